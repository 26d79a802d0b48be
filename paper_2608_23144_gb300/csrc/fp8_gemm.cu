// fp8_gemm.cu — y = x w^T for two matrices held in e4m3 codes with one
// power-of-two scale per row and 128 columns, on the fifth-generation tensor cores:
// the choice between two kernels, and the one for few rows of x.
//
// Mathematics: y[t][i] = sum_b 2^(ex[t][b] + ew[i][b]) sum_{k in b} cx[t][k] cw[i][k].
// The scales are powers of two, so the tensor cores apply them
// (kind::mxf8f6f4, scales of 8 exponent bits): one scale stands for four groups of
// 32 columns, the same byte for each of a block's four products.
//
// Few rows of x (up to 64: single tokens, drafts): the bytes of w bound it. A tile is
// 128 rows of w (tensor memory's lanes) x N rows of x (columns). Warp 8 copies: both
// matrices lie in memory as the tensor cores read them (rows of 128 bytes, their
// 16-byte pieces exchanged by row), so a block's rows are one bulk copy each, and a
// ring of stages as deep as shared memory keeps 200 KB per SM in flight. Rows of w
// start on their way while x is still being quantised. Warp 9 issues the products,
// warps 0-7 read the sums and write y. Few tiles: a cluster shares a tile's columns
// and joins its parts, in their order, through shared memory.
//
// Every wait is bounded (wait_ns): one that runs out sets bit 2 of the fault word,
// stops the block's roles, waits (bounded) for its copies and products in flight
// and frees the tensor memory.
#include "fp8_mma.cuh"
#include "internal.h"

namespace awsrc {

namespace {

using namespace fp8;

constexpr int kMaxSplit = 8;  // thread blocks that share a tile's columns
constexpr int kLeast = 4;     // blocks that one of them has at least

template <int N>
struct Cfg {
  static constexpr int kStageBytes = (BM + N) * 128;
  static constexpr int kStages = N > 32 ? 8 : N > 16 ? 10 : 11;
  static constexpr int kAccCols = 2 * N;  // two accumulators
  static constexpr int kSfCols = 8;       // a set of scales: 4 columns for w, 4 for x
  static constexpr int kCols = kAccCols + kSfSets * kSfCols;
  static constexpr int kTmem = kCols > 128 ? 256 : 128;
  static constexpr int kPer = N / 2;  // columns of an epilogue thread
};

template <int N>
struct Smem {
  using C = Cfg<N>;
  uint8_t tile[C::kStages][C::kStageBytes];
  uint8_t sf[C::kStages][1024];  // scales of w, of x
  unsigned long long full[C::kStages], empty[C::kStages], acc_full[2], acc_empty[2], drain;
  uint32_t tmem;
  int dead;
};

__device__ __forceinline__ void copy_sf(uint32_t taddr, uint64_t desc) {  // 512 bytes to 4 columns, in all lanes' quarters
  asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc) : "memory");
}
__device__ __forceinline__ void umma_mx(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sfa, uint32_t sfb,
                                        uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %6, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale [%0], %1, %2, %3, [%4], [%5], p;\n\t}" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate)
      : "memory");
}

// The walk that all roles take: tiles of this block, its share of their columns in
// chunks of blocks.
struct Walk {
  int tiles, chunk, step;
  int tile, lo, hi, k0, k1;
  __device__ Walk(const GemmArgs& a, bool f32) {
    tiles = a.w.tiles();  // one tile of rows of x
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
  __device__ void next() {
    if (last()) tile += step, k0 = lo;
    else k0 = k1;
    k1 = min(k0 + chunk, hi);
  }
};

template <int N, bool kF32>
__device__ void copy_role(const GemmArgs& a, Smem<N>& sm, const Ctx& x) {
  using C = Cfg<N>;
  const int lane = threadIdx.x & 31;
  const int64_t w8 = a.w.rows8(), x8 = a.x.rows8();
  const uint32_t xb = 128u * (uint32_t)x8;
  bool ok = true;
  Walk w(a, kF32);
  const auto has_sf = [&](int kb) { return (kb & 3) == 0 || kb == w.lo; };
  const auto copy_w = [&](int kb, uint32_t s) {  // block kb of the tile to stage s: what comes of w
    const int row = w.tile * BM;
    const uint32_t wb = 128u * (uint32_t)min((int64_t)BM, w8 - row);
    mbar_expect_tx(&sm.full[s], wb + xb + (has_sf(kb) ? 1024u : 0u));
    bulk_g2s(sm.tile[s], a.w.codes + (kb * w8 + row) * 128, wb, &sm.full[s]);
    if (has_sf(kb)) bulk_g2s(sm.sf[s], a.w.exps + ((int64_t)(kb >> 2) * a.w.tiles() + w.tile) * 512, 512, &sm.full[s]);
  };
  const auto copy_x = [&](int kb, uint32_t s) {
    bulk_g2s(sm.tile[s] + BM * 128, a.x.codes + kb * x8 * 128, xb, &sm.full[s]);
    if (has_sf(kb)) bulk_g2s(sm.sf[s] + 512, a.x.exps + (int64_t)(kb >> 2) * 512, 512, &sm.full[s]);
  };
  // the first blocks fill the stages, a lane each; rows of w are on their way before x is ready
  int ahead = w.more() ? min(C::kStages, w.hi - w.lo) : 0;
  if (a.stall >= 0) ahead = 0;
  if (a.early && lane < ahead) copy_w(w.lo + lane, lane);
  step_wait();
  if (lane < ahead) {
    if (!a.early) copy_w(w.lo + lane, lane);
    copy_x(w.lo + lane, lane);
  }
  __syncwarp();
  uint32_t n = 0;             // blocks so far
  uint32_t s = 0, phase = 1;  // stage of block n
  const int64_t w_step = w8 * 128, x_step = x8 * 128;
  for (; ok && w.more(); w.next()) {
    const int row = w.tile * BM;
    const uint32_t wb = 128u * (uint32_t)min((int64_t)BM, w8 - row);
    const uint8_t *wp = a.w.codes + w.k0 * w_step + row * 128ll, *xp = a.x.codes + w.k0 * x_step;
    for (int kb = w.k0; kb < w.k1; ++kb, ++n, wp += w_step, xp += x_step) {
      if ((int)n >= ahead) {
        if (kb == a.stall || !wait_warp(x, &sm.empty[s], phase)) {
          ok = false;
          break;
        }
        const bool sf = has_sf(kb);
        const uint8_t *ws = a.w.exps + ((int64_t)(kb >> 2) * a.w.tiles() + w.tile) * 512, *xs = a.x.exps + (int64_t)(kb >> 2) * 512;
        if (one_lane()) {
          mbar_expect_tx(&sm.full[s], wb + xb + (sf ? 1024u : 0u));
          bulk_g2s(sm.tile[s], wp, wb, &sm.full[s]);
          bulk_g2s(sm.tile[s] + BM * 128, xp, xb, &sm.full[s]);
          if (sf) {
            bulk_g2s(sm.sf[s], ws, 512, &sm.full[s]);
            bulk_g2s(sm.sf[s] + 512, xs, 512, &sm.full[s]);
          }
        }
        __syncwarp();
      }
      if (++s == C::kStages) s = 0, phase ^= 1;
    }
  }
  if (!ok)  // copies in flight land before the block ends
    for (uint32_t j = n > C::kStages ? n - C::kStages : 0; j < n; ++j)
      (void)mbar_wait(&sm.full[j % C::kStages], (j / C::kStages) & 1, x.wait_ns);
}

template <int N, bool kF32>
__device__ void mma_role(const GemmArgs& a, Smem<N>& sm, const Ctx& x, uint32_t tmem) {
  using C = Cfg<N>;
  uint32_t n = 0, c = 0;      // blocks, chunks so far
  uint32_t s = 0, phase = 0;  // stage of block n
  SfSets sets;
  bool ok = true;
  const uint32_t idesc0 = idesc_mx(BM, N);
  const uint64_t tile0 = desc_rows(smem_addr(sm.tile[0])), sf0 = desc_sf(smem_addr(sm.sf[0]));
  for (Walk w(a, kF32); ok && w.more(); w.next(), ++c) {
    const uint32_t buf = c & 1, d = tmem + buf * N;
    uint32_t sfa = tmem + C::kAccCols + sets.at() * C::kSfCols;
    if (!(ok = wait_warp(x, &sm.acc_empty[buf], ((c >> 1) & 1) ^ 1))) break;
    tc_fence_after();
    for (int kb = w.k0; kb < w.k1; ++kb, ++n) {
      if (!(ok = wait_warp(x, &sm.full[s], phase))) break;
      tc_fence_after();
      const bool sf = (kb & 3) == 0 || kb == w.lo;
      if (sf) {
        if (!(ok = sets.open<C::kStages, 1>(x, sm.empty, n))) break;
        sfa = tmem + C::kAccCols + sets.at() * C::kSfCols;
      }
      const uint64_t ds = sf0 + s * (1024 / 16);
      const uint32_t idesc = with_sf_id(idesc0, kb & 3);
      const uint64_t da = tile0 + s * (C::kStageBytes / 16), db = da + BM * 128 / 16;
      if (one_lane()) {
        if (sf) {
          copy_sf(sfa, ds);
          copy_sf(sfa + 4, ds + 32);
        }
        umma_mx(d, da, db, idesc, sfa, sfa + 4, kb != w.k0);
#pragma unroll
        for (int j = 1; j < 4; ++j) umma_mx(d, da + 2 * j, db + 2 * j, idesc, sfa, sfa + 4, 1);
        umma_commit(&sm.empty[s]);
        if (kb + 1 == w.k1) umma_commit(&sm.acc_full[buf]);
      }
      __syncwarp();
      if (++s == C::kStages) s = 0, phase ^= 1;
    }
  }
  if (!ok && one_lane()) {  // products in flight end before the block does
    umma_commit(&sm.drain);
    (void)mbar_wait(&sm.drain, 0, x.wait_ns);
  }
}

template <int N, bool kF32>
__device__ void write_role(const GemmArgs& a, Smem<N>& sm, const Ctx& x, uint32_t tmem) {
  using C = Cfg<N>;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t quarter = warp & 3, c0 = (warp >> 2) * C::kPer;
  float acc[C::kPer];
  uint32_t c = 0;
  for (Walk w(a, kF32); w.more(); w.next(), ++c) {
    const uint32_t buf = c & 1;
    if (!wait_warp(x, &sm.acc_full[buf], (c >> 1) & 1)) return;
    tc_fence_after();
    const uint32_t t = tmem + ((quarter * 32) << 16) + buf * N + c0;
    float v[C::kPer];
#pragma unroll
    for (int i = 0; i < C::kPer; i += 8) tmem_ld8(t + i, v + i);
    tmem_wait_ld8(v);
#pragma unroll
    for (int i = 8; i < C::kPer; i += 8) tmem_tie8(v + i);
#pragma unroll
    for (int i = 0; i < C::kPer; ++i) acc[i] = kF32 && !w.first() ? __fadd_rn(acc[i], v[i]) : v[i];
    tc_fence_before();
    mbar_arrive(&sm.acc_empty[buf]);
    if (!w.last()) continue;
    const int r = quarter * 32 + lane, row = w.tile * BM + r;
    if (a.split > 1) {  // the part stays here until the cluster joins it; all copies and products of the block are done
      float* part = reinterpret_cast<float*>(sm.tile[0]);
#pragma unroll
      for (int i = 0; i < C::kPer; ++i) part[(c0 + i) * BM + r] = acc[i];
    } else if (row < a.w.rows) {
#pragma unroll
      for (int i = 0; i < C::kPer; ++i)
        if ((int)c0 + i < a.x.rows) put<kF32>(a, c0 + i, row, acc[i]);
    }
  }
}

// The cluster's parts of a tile joined; each thread block joins its share of the elements.
template <int N, bool kF32>
__device__ void join(const GemmArgs& a, Smem<N>& sm) {
  const int rank = blockIdx.x % a.split, row0 = blockIdx.x / a.split * BM;
  for (int e = rank * kThreads + threadIdx.x; e < a.x.rows * (BM / 4); e += a.split * kThreads)
    put4<kF32>(a, e / (BM / 4), row0 + e % (BM / 4) * 4, join4(smem_addr(sm.tile[0]) + 16 * e, 0, 1, a.split));
}

template <int N, bool kF32>
__global__ void __launch_bounds__(kThreads, 1) fp8_few_kernel(const __grid_constant__ GemmArgs a) {
  using C = Cfg<N>;
  extern __shared__ unsigned char smem_raw[];
  Smem<N>& sm = *reinterpret_cast<Smem<N>*>(smem_raw + ((1024u - (smem_addr(smem_raw) & 1023u)) & 1023u));
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
  } else if (warp == kCopyWarp) {
    copy_role<N, kF32>(a, sm, x);
  } else {
    mma_role<N, kF32>(a, sm, x, tmem);
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
  using C = Cfg<N>;
  constexpr int kSmem = (int)sizeof(Smem<N>) + 1024;
  static_assert(kSmem <= 227 * 1024, "shared memory of a block");
  static_assert(N * BM * 4 <= C::kStages * C::kStageBytes, "a part of a tile fits into the stages");
  const cudaError_t e = cudaFuncSetAttribute(fp8_few_kernel<N, kF32>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
  if (e != cudaSuccess) return e;
  GemmArgs a = in;
  const int tiles = a.w.tiles(), slots = 152, blocks = a.x.blocks();
  // few tiles: the columns of each are split over a cluster, at least kLeast blocks each
  a.split = slots / tiles;
  if (a.split > kMaxSplit) a.split = kMaxSplit;
  if (a.split > blocks / kLeast) a.split = blocks / kLeast;
  if (a.split < 1) a.split = 1;
  const int grid = a.split > 1 ? tiles * a.split : tiles < slots ? tiles : slots;
  return launch_step(fp8_few_kernel<N, kF32>, dim3((unsigned)grid), kThreads, kSmem, a.split, st, a);
}

}  // namespace

cudaError_t launch_fp8_gemm(const GemmArgs& in, int y_dtype, cudaStream_t st) {
  const bool f32 = y_dtype == AWSRC_DTYPE_F32;
  GemmArgs a = in;
  const uintptr_t size = f32 ? 4 : 2;
  a.vec_y = (reinterpret_cast<uintptr_t>(a.y) | (uintptr_t)a.ys * size) % (4 * size) == 0;
  cudaError_t e;
  if (a.x.rows <= 16) e = f32 ? launch<16, true>(a, st) : launch<16, false>(a, st);
  else if (a.x.rows <= 32) e = f32 ? launch<32, true>(a, st) : launch<32, false>(a, st);
  else if (a.x.rows <= 64) e = f32 ? launch<64, true>(a, st) : launch<64, false>(a, st);
  else e = launch_fp8_pairs(a, f32, st);
  if (e != cudaSuccess) return e;
  note_launches(1);
  return cudaGetLastError();
}

}  // namespace awsrc
