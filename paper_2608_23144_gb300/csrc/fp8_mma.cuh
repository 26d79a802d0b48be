// fp8_mma.cuh — what the kernels of 8-bit products share: bounded waits,
// descriptors of operands and scales, results.
#pragma once

#include <cuda.h>

#include "fp8_choice.h"
#include "step.cuh"
#include "tc05.cuh"

namespace awsrc {

// Clusters of thread blocks, one per SM, that the current device runs at a time (fewer than
// its SMs allow: a cluster lies in one group of them). An answer is kept, a failure is the
// call's: with other shares the sums would have another order.
cudaError_t max_clusters(fp8::Clusters* most);

// A tiled tensor of up to 3 dimensions (innermost first), rows past the last read as 0.
cudaError_t make_tensor_map(CUtensorMap* map, CUtensorMapDataType type, int rank, const void* p, const cuuint64_t* dims,
                            const cuuint64_t* strides, const cuuint32_t* box);

namespace fp8 {

using namespace tc05;

constexpr int BM = kTileRows;
// Blocks summed in tensor memory before the sums leave it: the cores cut a running sum off
// (below 2^-24 of it, measured) at each of a block's four products. Positive terms are off by
// 3e-7 after 2048 columns and 1.2e-5 after 27648; bf16 results are rounded by up to 2^-8 of their own.
constexpr int kChunkF32 = 16, kChunkBf16 = 256;

struct Ctx {
  uint64_t wait_ns;
  uint32_t* status;
  volatile int* dead;
};

// Bounded wait; false once any wait of the block has given up.
static __device__ __noinline__ bool wait_slow(const Ctx& x, unsigned long long* mb, uint32_t parity) {
  const uint64_t t0 = globaltimer();
  for (;;) {
    if (mbar_try_wait(mb, parity)) return true;
    if (*x.dead) return false;
    if (globaltimer() - t0 > x.wait_ns) {
      *x.dead = 1;
      atomicOr(x.status, kFaultTimeout);
      return false;
    }
  }
}
__device__ __forceinline__ bool wait_lane(const Ctx& x, unsigned long long* mb, uint32_t parity) {
  return mbar_try_wait(mb, parity) || wait_slow(x, mb, parity);
}
__device__ __forceinline__ bool wait_warp(const Ctx& x, unsigned long long* mb, uint32_t parity) {
  return __all_sync(0xffffffffu, wait_lane(x, mb, parity));
}

// One lane of a converged warp. The products' warp runs as a whole, so that what its
// instructions take is computed once per warp, and one lane issues them: a lane that
// ran alone took 340 ns a block, whatever the products.
__device__ __forceinline__ bool one_lane() {
  uint32_t r;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(r));
  return r != 0;
}

// Scales of 4 blocks lie in tensor memory in one of 4 sets, used in turn. Set k + 4
// overwrites set k, whose products must be done: with 4 blocks a set they are, as the
// ring of stages has been around since (13 blocks lie between, kMaxStages is no more);
// where tiles or shares end early, the products of set k's last block are waited for.
constexpr int kSfSets = 4, kMaxStages = 13;
struct SfSets {
  uint32_t count = 0, o1 = 0, o2 = 0, o3 = 0;  // sets so far; first blocks of the last three
  // Opens the set of block n; false once a wait has given up. empty[] has a barrier for
  // each kPer stages, told after the last of their blocks (at least 4 lie between).
  template <int kStages, int kPer>
  __device__ __forceinline__ bool open(const Ctx& x, unsigned long long* empty, uint32_t n) {
    static_assert(kStages <= kMaxStages - (kPer - 1), "a set's products are done when it is used again");
    static_assert(kPer <= 4, "a set's last products have been told of");
    bool ok = true;
    if (count >= kSfSets && n - (o3 - 1) < kStages) {
      const uint32_t last = o3 - 1;
      ok = wait_warp(x, &empty[last % kStages / kPer], (last / kStages) & 1);
    }
    o3 = o2;
    o2 = o1;
    o1 = n;
    ++count;
    return ok;
  }
  __device__ __forceinline__ uint32_t at() const { return (count - 1) % kSfSets; }
};

// Whether the phase is over, without waiting: asked ahead, its answer comes while products are issued.
__device__ __forceinline__ bool mbar_test(unsigned long long* mb, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok)
      : "r"(smem_addr(mb)), "r"(parity)
      : "memory");
  return ok != 0;
}

// Rows of 128 bytes, 16-byte pieces exchanged by row (128-byte swizzle), groups of
// 8 rows 1024 bytes apart.
__device__ __forceinline__ uint64_t desc_rows(uint32_t addr) {
  return (uint64_t)((addr & 0x3FFFFu) >> 4) | (1ull << 16) | ((uint64_t)(1024u >> 4) << 32) | (1ull << 46) | (2ull << 61);
}
// 32 rows of 16 bytes: what a copy of scales to tensor memory reads.
__device__ __forceinline__ uint64_t desc_sf(uint32_t addr) {
  return (uint64_t)((addr & 0x3FFFFu) >> 4) | (1ull << 16) | ((uint64_t)(128u >> 4) << 32) | (1ull << 46);
}
// Byte `id` of the scale words is the one to use.
__device__ __forceinline__ uint32_t with_sf_id(uint32_t idesc, uint32_t id) { return idesc | (id << 4) | (id << 29); }

// e4m3 x e4m3, scales of 8 exponent bits, one per 32 columns; M rows of w, n of x.
__device__ __forceinline__ uint32_t idesc_mx(int m, int n) {
  return (1u << 23) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}

__device__ __forceinline__ void put(const GemmArgs& a, int tok, int row, float v) {
  const int64_t at = (int64_t)tok * a.ys + row;
  if (a.y_f32) static_cast<float*>(a.y)[at] = v;
  else static_cast<__nv_bfloat16*>(a.y)[at] = __float2bfloat16_rn(v);
}

// Four columns of a lane's row become four rows of a column: of lanes 4 a .. 4 a + 3, lane
// 4 a + b gets column b. A store instruction takes 9 cycles however little of it there is
// (results of one column a warp, 64 or 128 bytes, took 150 us where 50 or 96 write as much).
__device__ __forceinline__ float4 quad(float r0, float r1, float r2, float r3) {
  const bool odd = threadIdx.x & 1, high = threadIdx.x & 2;
  const float s = __shfl_xor_sync(0xffffffffu, odd ? r0 : r1, 1), t = __shfl_xor_sync(0xffffffffu, odd ? r2 : r3, 1);
  r0 = odd ? s : r0;
  r1 = odd ? r1 : s;
  r2 = odd ? t : r2;
  r3 = odd ? r3 : t;
  const float u = __shfl_xor_sync(0xffffffffu, high ? r0 : r2, 2), v = __shfl_xor_sync(0xffffffffu, high ? r1 : r3, 2);
  return high ? make_float4(u, v, r2, r3) : make_float4(r0, r1, u, v);
}

// Four floats at `addr` in the shared memory of each of `split` thread blocks, rank0
// being the first and `every` the step between them. (25 GB/s from a partner.)
template <int kSplit>
__device__ __forceinline__ void get_parts(float4* v, uint32_t addr, int rank0, int every, int split) {
#pragma unroll
  for (int z = 0; z < kSplit; ++z)
    if (z < split) {
      uint32_t peer;
      asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(peer) : "r"(addr), "r"(rank0 + z * every));
      asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
                   : "=f"(v[z].x), "=f"(v[z].y), "=f"(v[z].z), "=f"(v[z].w) : "r"(peer) : "memory");
    }
}
template <int kSplit>
__device__ __forceinline__ float4 sum_parts(const float4* v, int split) {
  float4 sum = v[0];
#pragma unroll
  for (int z = 1; z < kSplit; ++z)
    if (z < split)
      sum = make_float4(__fadd_rn(sum.x, v[z].x), __fadd_rn(sum.y, v[z].y), __fadd_rn(sum.z, v[z].z), __fadd_rn(sum.w, v[z].w));
  return sum;
}

// Four rows of w of one row of y.
__device__ __forceinline__ void put4(const GemmArgs& a, int tok, int row, float4 v) {
  const int have = a.w.rows - row;
  if (have >= 4 && a.vec_y) {
    const int64_t at = (int64_t)tok * a.ys + row;
    if (a.y_f32) {
      *reinterpret_cast<float4*>(static_cast<float*>(a.y) + at) = v;
    } else {
      const __nv_bfloat162 lo = __floats2bfloat162_rn(v.x, v.y), hi = __floats2bfloat162_rn(v.z, v.w);
      *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(a.y) + at) =
          make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi));
    }
    return;
  }
  if (have > 0) put(a, tok, row, v.x);
  if (have > 1) put(a, tok, row + 1, v.y);
  if (have > 2) put(a, tok, row + 2, v.z);
  if (have > 3) put(a, tok, row + 3, v.w);
}

}  // namespace fp8
}  // namespace awsrc
