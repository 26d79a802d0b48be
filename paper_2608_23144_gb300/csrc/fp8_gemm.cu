// fp8_gemm.cu — y = x w^T for two matrices held in e4m3 codes with one
// power-of-two scale per row and 128 columns, on the fifth-generation tensor cores.
//
// Mathematics: y[t][i] = sum_b 2^(ex[t][b] + ew[i][b]) sum_{k in b} cx[t][k] cw[i][k].
// The scales are powers of two, so the tensor cores apply them
// (kind::mxf8f6f4, scales of 8 exponent bits): one scale stands for four groups of
// 32 columns, the same byte for each of a block's four products.
//
// A tile is 128 rows of w (tensor memory's lanes) x N rows of x (columns). Warp 8
// copies: both matrices lie in memory as the tensor cores read them (rows of 128
// bytes, their 16-byte pieces exchanged by row), so a block's rows are one bulk
// copy each. Warp 9 issues the products. Warps 0-7 read the sums and write y.
//
// Every wait is bounded (wait_ns): one that runs out sets bit 2 of the fault word,
// stops the block's roles, waits (bounded) for its copies and products in flight
// and frees the tensor memory.
#include "internal.h"
#include "step.cuh"
#include "tc05.cuh"

namespace awsrc {

namespace {

using namespace tc05;

constexpr int BM = 128;
constexpr int kThreads = 320, kCopyWarp = 8, kMmaWarp = 9;
constexpr int kSfSets = 4;    // scales of 4 blocks each in tensor memory; more ahead than stages
constexpr int kChunk = 16;    // blocks summed in tensor memory for F32 results
constexpr int kMaxSplit = 8;  // thread blocks that share a tile's columns
constexpr int kLeast = 4;     // blocks that one of them has at least

template <int N, bool kF32>
struct Cfg {
  static constexpr int kXRows = N;
  static constexpr int kStageBytes = (BM + N) * 128;
  static constexpr int kXSf = N > 128 ? 2 : 1;  // 512-byte scale tiles of x
  static constexpr int kSfBytes = 512 * (1 + kXSf);
  static constexpr int kBufs = N > 128 ? 1 : 2;  // accumulators
  static constexpr int kPerSm = N > 64 ? 1 : 2;  // thread blocks
  static constexpr int kStages = N > 128 ? 4 : N > 64 ? 6 : N > 32 ? 4 : 5;
  static constexpr int kAccCols = kBufs * N;
  static constexpr int kSfCols = 4 * (1 + kXSf);
  static constexpr int kCols = kAccCols + kSfSets * kSfCols;
  static constexpr int kTmem = kCols > 256 ? 512 : kCols > 128 ? 256 : 128;
  static constexpr int kPer = N / 2;  // columns of an epilogue thread
};

template <int N, bool kF32>
struct Smem {
  using C = Cfg<N, kF32>;
  uint8_t tile[C::kStages][C::kStageBytes];
  uint8_t sf[C::kStages][C::kSfBytes];
  unsigned long long full[C::kStages], empty[C::kStages], acc_full[2], acc_empty[2], drain;
  uint32_t tmem;
  int dead;
};

struct Ctx {
  uint64_t wait_ns;
  uint32_t* status;
  volatile int* dead;
};

// Bounded wait; false once any wait of the block has given up.
__device__ __noinline__ bool wait_slow(const Ctx& x, unsigned long long* mb, uint32_t parity) {
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

// Rows of 128 bytes, 16-byte pieces exchanged by row (128-byte swizzle), groups of
// 8 rows 1024 bytes apart.
__device__ __forceinline__ uint64_t desc_rows(uint32_t addr) {
  return (uint64_t)((addr & 0x3FFFFu) >> 4) | (1ull << 16) | ((uint64_t)(1024u >> 4) << 32) | (1ull << 46) | (2ull << 61);
}
// 32 rows of 16 bytes: what a copy of scales to tensor memory reads.
__device__ __forceinline__ uint64_t desc_sf(uint32_t addr) {
  return (uint64_t)((addr & 0x3FFFFu) >> 4) | (1ull << 16) | ((uint64_t)(128u >> 4) << 32) | (1ull << 46);
}
// 512 bytes of scales to 4 columns, in all four quarters of the lanes.
__device__ __forceinline__ void copy_sf(uint32_t taddr, uint64_t desc) {
  asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc) : "memory");
}

// e4m3 x e4m3, scales of 8 exponent bits, one per 32 columns; rows in D's lanes: w.
template <int N>
struct IdescMx {
  static constexpr uint32_t value = (1u << 23) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(BM >> 4) << 24);
};
// Byte `id` of the scale words is the one to use.
__device__ __forceinline__ uint32_t with_sf_id(uint32_t idesc, uint32_t id) { return idesc | (id << 4) | (id << 29); }

__device__ __forceinline__ void umma_mx(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sfa, uint32_t sfb,
                                        uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %6, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale [%0], %1, %2, %3, [%4], [%5], p;\n\t}" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate)
      : "memory");
}

// The walk that all roles take: tiles of this block, in chunks of blocks.
struct Walk {
  int tiles_w, tiles, chunk, step;
  int tile, lo, hi, k0, k1;
  __device__ Walk(const GemmArgs& a, int n, bool f32) {
    tiles_w = a.w.tiles();
    tiles = tiles_w * ((a.x.rows + n - 1) / n);
    const int blocks = a.x.blocks(), rank = blockIdx.x % a.split;
    step = gridDim.x / a.split;
    tile = blockIdx.x / a.split;
    lo = (int)((int64_t)blocks * rank / a.split);
    hi = (int)((int64_t)blocks * (rank + 1) / a.split);
    chunk = f32 ? kChunk : blocks;
    k0 = lo;
    k1 = min(k0 + chunk, hi);
  }
  __device__ bool more() const { return tile < tiles; }
  __device__ bool first() const { return k0 == lo; }
  __device__ bool last() const { return k1 == hi; }
  __device__ int row() const { return tile % tiles_w * BM; }
  __device__ int tok(int n) const { return tile / tiles_w * n; }
  __device__ void next() {
    if (last()) tile += step, k0 = lo;
    else k0 = k1;
    k1 = min(k0 + chunk, hi);
  }
};

template <int N, bool kF32>
__device__ void copy_role(const GemmArgs& a, Smem<N, kF32>& sm, const Ctx& x) {
  using C = Cfg<N, kF32>;
  const int64_t w8 = a.w.rows8(), x8 = a.x.rows8();
  uint32_t n = 0;
  int ahead = 0;  // blocks whose rows of w are on their way before x is ready
  bool ok = true;
  Walk w(a, N, kF32);
  // block kb of the tile to stage s: what comes of w, then what comes of x
  const auto begin = [&](int kb, uint32_t s) {
    const int row = w.row(), tok = w.tok(N);
    const bool sf = (kb & 3) == 0 || kb == w.lo;
    const uint32_t wb = 128u * (uint32_t)min((int64_t)BM, w8 - row), xb = 128u * (uint32_t)min((int64_t)N, x8 - tok);
    const uint32_t xs = 512u * (uint32_t)min(C::kXSf, a.x.tiles() - (tok >> 7));
    mbar_expect_tx(&sm.full[s], wb + xb + (sf ? 512u + xs : 0u));
    bulk_g2s(sm.tile[s], a.w.codes + (kb * w8 + row) * 128, wb, &sm.full[s]);
    if (sf) bulk_g2s(sm.sf[s], a.w.exps + ((int64_t)(kb >> 2) * a.w.tiles() + (row >> 7)) * 512, 512, &sm.full[s]);
  };
  const auto finish = [&](int kb, uint32_t s) {
    const int tok = w.tok(N);
    const uint32_t xb = 128u * (uint32_t)min((int64_t)N, x8 - tok);
    bulk_g2s(sm.tile[s] + BM * 128, a.x.codes + (kb * x8 + tok) * 128, xb, &sm.full[s]);
    if ((kb & 3) == 0 || kb == w.lo)
      bulk_g2s(sm.sf[s] + 512, a.x.exps + ((int64_t)(kb >> 2) * a.x.tiles() + (tok >> 7)) * 512,
               512u * (uint32_t)min(C::kXSf, a.x.tiles() - (tok >> 7)), &sm.full[s]);
  };
  if (a.early && a.stall < 0 && w.more())
    for (; ahead < min(C::kStages, w.hi - w.lo); ++ahead) begin(w.lo + ahead, ahead);
  step_wait();
  for (; ok && w.more(); w.next()) {
    for (int kb = w.k0; kb < w.k1; ++kb, ++n) {
      const uint32_t s = n % C::kStages;
      if ((int)n >= ahead) {
        if (kb == a.stall || !wait_lane(x, &sm.empty[s], ((n / C::kStages) & 1) ^ 1)) {
          ok = false;
          break;
        }
        begin(kb, s);
      }
      finish(kb, s);
    }
  }
  if (!ok)  // copies in flight land before the block ends
    for (uint32_t j = n > C::kStages ? n - C::kStages : 0; j < n; ++j)
      (void)mbar_wait(&sm.full[j % C::kStages], (j / C::kStages) & 1, x.wait_ns);
}

template <int N, bool kF32>
__device__ void mma_role(const GemmArgs& a, Smem<N, kF32>& sm, const Ctx& x, uint32_t tmem) {
  using C = Cfg<N, kF32>;
  uint32_t n = 0, c = 0, g = 0;  // blocks, chunks, scale sets so far
  bool ok = true;
  for (Walk w(a, N, kF32); ok && w.more(); w.next(), ++c) {
    const uint32_t buf = c % C::kBufs;
    if (!(ok = wait_lane(x, &sm.acc_empty[buf], ((c / C::kBufs) & 1) ^ 1))) break;
    tc_fence_after();
    for (int kb = w.k0; kb < w.k1; ++kb, ++n) {
      const uint32_t s = n % C::kStages;
      if (!(ok = wait_lane(x, &sm.full[s], (n / C::kStages) & 1))) break;
      tc_fence_after();
      if ((kb & 3) == 0 || kb == w.lo) {
        ++g;
        const uint32_t at = tmem + C::kAccCols + (g % kSfSets) * C::kSfCols;
#pragma unroll
        for (int i = 0; i < 1 + C::kXSf; ++i) copy_sf(at + 4 * i, desc_sf(smem_addr(sm.sf[s] + 512 * i)));
      }
      const uint32_t sfa = tmem + C::kAccCols + (g % kSfSets) * C::kSfCols, sfb = sfa + 4;
      const uint32_t idesc = with_sf_id(IdescMx<N>::value, kb & 3);
      const uint64_t da = desc_rows(smem_addr(sm.tile[s])), db = desc_rows(smem_addr(sm.tile[s] + BM * 128));
#pragma unroll
      for (int j = 0; j < 4; ++j)
        umma_mx(tmem + buf * N, da + 2 * j, db + 2 * j, idesc, sfa, sfb, kb != w.k0 || j != 0);
      umma_commit(&sm.empty[s]);
    }
    if (ok) umma_commit(&sm.acc_full[buf]);
  }
  if (!ok) {  // products in flight end before the block does
    umma_commit(&sm.drain);
    (void)mbar_wait(&sm.drain, 0, x.wait_ns);
  }
}

template <bool kF32>
__device__ __forceinline__ void put(const GemmArgs& a, int tok, int row, float v) {
  const int64_t at = (int64_t)tok * a.ys + row;
  if (kF32) static_cast<float*>(a.y)[at] = v;
  else static_cast<__nv_bfloat16*>(a.y)[at] = __float2bfloat16_rn(v);
}

// Sums of this thread's row and columns; false once a wait has given up.
template <int N, bool kF32>
__device__ bool write_role(const GemmArgs& a, Smem<N, kF32>& sm, const Ctx& x, uint32_t tmem) {
  using C = Cfg<N, kF32>;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t quarter = warp & 3, c0 = (warp >> 2) * C::kPer;
  float acc[C::kPer];
  uint32_t c = 0;
  for (Walk w(a, N, kF32); w.more(); w.next(), ++c) {
    const uint32_t buf = c % C::kBufs;
    if (!wait_warp(x, &sm.acc_full[buf], (c / C::kBufs) & 1)) return false;
    tc_fence_after();
    const uint32_t t = tmem + ((quarter * 32) << 16) + buf * N + c0;
#pragma unroll
    for (int i = 0; i < C::kPer; i += 8) {
      float v[8];
      tmem_ld8(t + i, v);
      tmem_wait_ld8(v);
#pragma unroll
      for (int j = 0; j < 8; ++j) acc[i + j] = kF32 && !w.first() ? __fadd_rn(acc[i + j], v[j]) : v[j];
    }
    tc_fence_before();
    mbar_arrive(&sm.acc_empty[buf]);
    if (!w.last()) continue;
    const int row = w.row() + quarter * 32 + lane, tok = w.tok(N) + c0;
    if (a.split > 1) {  // the part stays here until the cluster joins it; all copies and products of the block are done
      float* part = reinterpret_cast<float*>(sm.tile[0]);
#pragma unroll
      for (int i = 0; i < C::kPer; ++i) part[(c0 + i) * BM + quarter * 32 + lane] = acc[i];
    } else if (row < a.w.rows) {
#pragma unroll
      for (int i = 0; i < C::kPer; ++i)
        if (tok + i < a.x.rows) put<kF32>(a, tok + i, row, acc[i]);
    }
  }
  return true;
}

// The cluster's parts of a tile, in shared memory, joined in the order of their
// columns of w; each thread block joins its share of the tile's elements.
template <int N, bool kF32>
__device__ void join(const GemmArgs& a, Smem<N, kF32>& sm) {
  const Walk w(a, N, kF32);
  const int rank = blockIdx.x % a.split, row0 = w.row(), tok0 = w.tok(N);
  const int cols = min(N, a.x.rows - tok0);
  for (int e = rank * kThreads + threadIdx.x; e < cols * BM; e += a.split * kThreads) {
    const int row = row0 + e % BM;
    const uint32_t at = smem_addr(sm.tile[0]) + 4 * e;
    float sum = 0.0f;
    for (int z = 0; z < a.split; ++z) {
      uint32_t peer;
      float v;
      asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(peer) : "r"(at), "r"(z));
      asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(peer) : "memory");
      sum = z ? __fadd_rn(sum, v) : v;
    }
    if (row < a.w.rows) put<kF32>(a, tok0 + e / BM, row, sum);
  }
}

template <int N, bool kF32>
__global__ void __launch_bounds__(kThreads, Cfg<N, kF32>::kPerSm) fp8_gemm_kernel(const __grid_constant__ GemmArgs a) {
  using C = Cfg<N, kF32>;
  extern __shared__ unsigned char smem_raw[];
  Smem<N, kF32>& sm = *reinterpret_cast<Smem<N, kF32>*>(smem_raw + ((1024u - (smem_addr(smem_raw) & 1023u)) & 1023u));
  const int warp = threadIdx.x >> 5;
  if (warp == kMmaWarp) {
    if ((threadIdx.x & 31) == 0) {
      for (int i = 0; i < C::kStages; ++i) mbar_init(&sm.full[i], 1), mbar_init(&sm.empty[i], 1);
      for (int i = 0; i < 2; ++i) mbar_init(&sm.acc_full[i], 1), mbar_init(&sm.acc_empty[i], 256);
      mbar_init(&sm.drain, 1);
      sm.dead = 0;
      asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncwarp();
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&sm.tmem)),
                 "r"(C::kTmem)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    tc_fence_before();
  }
  __syncthreads();
  tc_fence_after();
  if (!a.early) step_wait();
  step_trigger();
  const Ctx x{a.wait_ns, a.status, &sm.dead};
  const uint32_t tmem = sm.tmem;
  if (warp < 8) {
    step_wait();
    write_role<N, kF32>(a, sm, x, tmem);
  } else if ((threadIdx.x & 31) == 0) {
    if (warp == kCopyWarp) copy_role<N, kF32>(a, sm, x);
    else mma_role<N, kF32>(a, sm, x, tmem);
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (warp == kMmaWarp) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(C::kTmem) : "memory");
  }
  if (a.split > 1) {  // every block gets here: all its waits are bounded
    __syncwarp();
    cluster_sync();
    join<N, kF32>(a, sm);
    __syncwarp();
    cluster_sync();  // no block leaves while others read its part
  }
}

template <int N, bool kF32>
cudaError_t launch(const GemmArgs& in, cudaStream_t st) {
  using C = Cfg<N, kF32>;
  constexpr int kSmem = (int)sizeof(Smem<N, kF32>) + 1024;
  static_assert(C::kPerSm * (kSmem + 1024) <= 228 * 1024, "shared memory of an SM");
  static_assert(N * BM * 4 <= C::kStages * C::kStageBytes, "a part of a tile fits into the stages");
  const cudaError_t e = cudaFuncSetAttribute(fp8_gemm_kernel<N, kF32>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
  if (e != cudaSuccess) return e;
  GemmArgs a = in;
  const int64_t tiles = (int64_t)a.w.tiles() * ((a.x.rows + N - 1) / N);
  const int slots = 152 * C::kPerSm, blocks = a.x.blocks();
  // few tiles: the columns of each are split over a cluster, at least kLeast blocks each
  a.split = (int)(slots / tiles);
  if (a.split > kMaxSplit) a.split = kMaxSplit;
  if (a.split > blocks / kLeast) a.split = blocks / kLeast;
  if (a.split < 1) a.split = 1;
  const int64_t grid = a.split > 1 ? tiles * a.split : tiles < slots ? tiles : slots;
  return launch_step(fp8_gemm_kernel<N, kF32>, dim3((unsigned)grid), kThreads, kSmem, a.split, st, a);
}

}  // namespace

cudaError_t launch_fp8_gemm(const GemmArgs& a, int y_dtype, cudaStream_t st) {
  const bool f32 = y_dtype == AWSRC_DTYPE_F32;
  cudaError_t e;
  if (a.x.rows <= 16) e = f32 ? launch<16, true>(a, st) : launch<16, false>(a, st);
  else if (a.x.rows <= 32) e = f32 ? launch<32, true>(a, st) : launch<32, false>(a, st);
  else if (a.x.rows <= 64) e = f32 ? launch<64, true>(a, st) : launch<64, false>(a, st);
  else if (f32 || a.x.rows <= 128 || (int64_t)a.w.tiles() * ((a.x.rows + 255) / 256) < 152)
    e = f32 ? launch<128, true>(a, st) : launch<128, false>(a, st);
  else e = launch<256, false>(a, st);
  if (e != cudaSuccess) return e;
  note_launches(1);
  return cudaGetLastError();
}

}  // namespace awsrc
