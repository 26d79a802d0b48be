// fp8_pairs.cu — y = x w^T for matrices held in 8 bits and more than 64 rows of x
// (chunks, prompts): mathematics and layouts as in fp8_gemm.cu, products by pairs of
// SMs (cta_group::2).
//
// Bound: a tile of 128 x 256 by one SM takes 48 KB per block of 128 columns, at the
// tensor cores' rate 96 bytes per cycle; the L2 gave 52, so such tiles ran at 55% of
// that rate. A pair's tile is 256 rows of w x n rows of x (64, 128, 192 or 256): each thread block brings 128 rows of w and half of the n rows of x, 32 KB per
// block, and its tensor core reads the other half from its partner.
//
// Roles in each thread block as in fp8_gemm.cu; the pair's even rank issues all
// products. Copies are of tensors, as only those can report to a partner's barrier:
// each thread block's count at the even rank's (a thread of the partner that waited
// for its own copies and passed it on took 950 cycles a block). One commit tells both
// that a stage is free, or the sums are ready; both tell the even rank when they have
// read them. Two accumulators where they fit beside the scales (n <= 192),
// so that one tile's results are read under the next one's products.
// Few tiles: a cluster of pairs shares a tile's columns and joins its parts.
//
// Measured: 8192 x 3584 x 18944 to bf16 318 to 336 us from one machine to the next, 3.3
// to 3.5 PFLOP/s or 85 to 90% of twice a large bf16 product's rate, to float32 375 (sums
// leave tensor memory every 2048 columns, results are twice the bytes); the tensor pipe is
// busy 71% of the cycles (2048 rows). Bound: the gap at a tile's end, where one
// accumulator of 256 columns has to be read (5%), commits, and under sustained load the
// power limit (2.8 PFLOP/s). 333 x 5000 x 1777 float32 11.6 us: 2.5 until the first
// product, 4 of products, 4 for parts that partners read at 25 GB/s.
//
// Every wait is bounded as in fp8_gemm.cu; no thread block of a cluster leaves before
// all have stopped, as products and arrivals reach into a partner's memory.
#include <atomic>

#include "fp8_mma.cuh"
#include "internal.h"

namespace awsrc {

namespace {

using namespace fp8;

constexpr int kThreads = 320, kCopyWarp = 8, kMmaWarp = 9;
constexpr int kMaxN = kPairMaxN;
constexpr int kStages = 6;
constexpr int kStageBytes = (BM + kMaxN / 2) * 128;
constexpr int kSfBytes = 512 * 3;  // scales of 128 rows of w, of up to 256 of x
constexpr int kSfCols = 12, kSfAt = 512 - kSfSets * kSfCols;
constexpr int kTwoBufs = 192;      // two accumulators of so many columns end before the scales
constexpr int kMaxSplit = kPairSplit;
constexpr int kGroup = 16;         // tiles of rows of x that are walked together (2: 354 us, 8: 332, 16: 325, 32: 333)

struct Smem {
  uint8_t tile[kStages][kStageBytes];
  uint8_t sf[kStages][kSfBytes];
  unsigned long long empty[kStages / 2], acc_full[2];
  unsigned long long full[kStages], acc_empty[2], drain;  // of the even rank
  uint32_t tmem;
  int dead;
};

// What the kernel takes: the codes as [block][row][128], the scales as [4 blocks][128
// rows][512 bytes]; rows past the last are read as 0.
struct PairArgs {
  CUtensorMap w_codes, x_codes, w_exps, x_exps;
  GemmArgs g;
};

// A box of a tensor to this thread block's shared memory; its bytes count at `mbar`, of either thread block of the pair.
__device__ __forceinline__ void copy_box(void* dst, const CUtensorMap* map, int row, int block, uint32_t mbar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(
          smem_addr(dst)),
      "l"(map), "r"(0), "r"(row), "r"(block), "r"(mbar)
      : "memory");
}

__device__ __forceinline__ uint32_t peer_addr(const void* p, uint32_t rank) {
  uint32_t r;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(smem_addr(p)), "r"(rank));
  return r;
}
// The default form: what has to be in order are reads of tensor memory, which tcgen05
// fences order. A release of the cluster's scope waits for the results stored before.
__device__ __forceinline__ void arrive_at(uint32_t mbar) {
  asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(mbar) : "memory");
}
// As mbar_try_wait, for arrivals from the partner.
__device__ __forceinline__ bool try_wait_cluster(unsigned long long* mb, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2, 20000;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok)
      : "r"(smem_addr(mb)), "r"(parity)
      : "memory");
  return ok != 0;
}
__device__ __forceinline__ bool mbar_test_cluster(unsigned long long* mb, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.test_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok)
      : "r"(smem_addr(mb)), "r"(parity)
      : "memory");
  return ok != 0;
}
__device__ __noinline__ bool wait_cluster_slow(const Ctx& x, unsigned long long* mb, uint32_t parity) {
  const uint64_t t0 = globaltimer();
  for (;;) {
    if (try_wait_cluster(mb, parity)) return true;
    if (*x.dead) return false;
    if (globaltimer() - t0 > x.wait_ns) {
      *x.dead = 1;
      atomicOr(x.status, kFaultTimeout);
      return false;
    }
  }
}
__device__ __forceinline__ bool wait_cluster(const Ctx& x, unsigned long long* mb, uint32_t parity) {
  return try_wait_cluster(mb, parity) || wait_cluster_slow(x, mb, parity);
}
__device__ __forceinline__ bool wait_cluster_warp(const Ctx& x, unsigned long long* mb, uint32_t parity) {
  return __all_sync(0xffffffffu, wait_cluster(x, mb, parity));
}

__device__ __forceinline__ void copy_sf(uint32_t taddr, uint64_t desc) {  // in both thread blocks, each from its own
  asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc) : "memory");
}
__device__ __forceinline__ void umma_mx(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sfa, uint32_t sfb,
                                        uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %6, 0;\n\t"
      "tcgen05.mma.cta_group::2.kind::mxf8f6f4.block_scale [%0], %1, %2, %3, [%4], [%5], p;\n\t}" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate)
      : "memory");
}
// Arrives at both thread blocks' barriers when the products so far are done.
__device__ __forceinline__ void commit_both(unsigned long long* mb, uint16_t mask) {
  asm volatile(
      "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(
          smem_addr(mb)),
      "h"(mask)
      : "memory");
}

// The walk that all roles take: tiles of this pair, its share of their columns in
// chunks of blocks. Tiles go by groups of kGroup tiles of rows of x, in a group by
// rows of w, so that what the pairs read together stays in the L2.
struct Walk {
  int tiles_w, tiles_x, tiles, chunk, step;
  int tile, lo, hi, k0, k1, row, tok;
  __device__ explicit Walk(const GemmArgs& a) {
    tiles_w = (a.w.tiles() + 1) >> 1;
    tiles_x = (a.x.rows + a.n - 1) / a.n;
    tiles = tiles_w * tiles_x;
    const unsigned pair = blockIdx.x >> 1, split = a.split, rank = pair % split, blocks = a.x.blocks();  // at most 2^17 blocks
    step = (gridDim.x >> 1) / split;
    tile = pair / split;
    lo = blocks * rank / split;
    hi = blocks * (rank + 1) / split;
    chunk = a.y_f32 ? kChunkF32 : kChunkBf16;
    k0 = lo;
    k1 = min(k0 + chunk, hi);
    place(a.n);
  }
  __device__ void place(int n) {
    const int g = tile / (kGroup * tiles_w) * kGroup, in = tile % (kGroup * tiles_w), many = min(kGroup, tiles_x - g);
    if (many < 1) return;  // past the last tile
    row = in / many * 2 * BM;
    tok = (g + in % many) * n;
  }
  __device__ bool more() const { return tile < tiles; }
  __device__ bool first() const { return k0 == lo; }
  __device__ bool last() const { return k1 == hi; }
  __device__ void next(int n) {
    if (last()) {
      tile += step;
      k0 = lo;
      place(n);
    } else {
      k0 = k1;
    }
    k1 = min(k0 + chunk, hi);
  }
};

// Scale tiles of 128 rows that the rows of x of a tile lie in.
__host__ __device__ constexpr int sf_tiles(int n) { return n > 128 ? 2 : 1; }

__device__ void copy_role(const PairArgs& p, Smem& sm, const Ctx& x, uint32_t half, uint32_t even) {
  const GemmArgs& a = p.g;
  uint32_t n = 0;
  int ahead;  // blocks whose copies begin together
  bool ok = true;
  Walk w(a);
  const int half_n = a.n >> 1;
  const uint32_t bytes = 2u * (BM * 128u + half_n * 128u), sf_bytes = 2u * 512u * (1 + sf_tiles(a.n));
  const auto has_sf = [&](int kb) { return (kb & 3) == 0 || kb == w.lo; };
  const auto copy_x = [&](int kb, uint32_t s) {
    const uint32_t mbar = peer_addr(&sm.full[s], even);
    copy_box(sm.tile[s] + BM * 128, &p.x_codes, w.tok + half_n * half, kb, mbar);
    if (has_sf(kb)) copy_box(sm.sf[s] + 512, &p.x_exps, w.tok >> 7, kb >> 2, mbar);
  };
  const auto copy_w = [&](int kb, uint32_t s) {  // what comes of w; the even rank's barrier counts both thread blocks' bytes
    const uint32_t mbar = peer_addr(&sm.full[s], even);
    if (!half) mbar_expect_tx(&sm.full[s], bytes + (has_sf(kb) ? sf_bytes : 0u));
    copy_box(sm.tile[s], &p.w_codes, w.row + BM * half, kb, mbar);
    if (has_sf(kb)) copy_box(sm.sf[s], &p.w_exps, (w.row >> 7) + half, kb >> 2, mbar);
  };
  // the first blocks fill the stages, a lane each; rows of w are on their way before x is ready
  const int lane = threadIdx.x & 31;
  ahead = w.more() && a.stall < 0 ? min(kStages, w.hi - w.lo) : 0;
  if (a.early && lane < ahead) copy_w(w.lo + lane, lane);
  step_wait();
  if (lane < ahead) {
    if (!a.early) copy_w(w.lo + lane, lane);
    copy_x(w.lo + lane, lane);
  }
  __syncwarp();
  uint32_t s = 0, phase = 1;  // stage of block n
  const uint32_t full0 = peer_addr(&sm.full[0], even);
  for (; ok && w.more(); w.next(a.n)) {
    const int row = w.row + BM * half, tok = w.tok + half_n * half;
    for (int kb = w.k0; kb < w.k1; ++kb, ++n) {
      if ((int)n >= ahead) {
        if (kb == a.stall || ((n & 1) == 0 && !wait_cluster_warp(x, &sm.empty[s >> 1], phase))) {
          ok = false;
          break;
        }
        const bool sf = has_sf(kb);
        const uint32_t mbar = full0 + 8 * s;
        if (one_lane()) {
          if (!half) mbar_expect_tx(&sm.full[s], bytes + (sf ? sf_bytes : 0u));
          copy_box(sm.tile[s], &p.w_codes, row, kb, mbar);
          copy_box(sm.tile[s] + BM * 128, &p.x_codes, tok, kb, mbar);
          if (sf) {
            copy_box(sm.sf[s], &p.w_exps, (w.row >> 7) + half, kb >> 2, mbar);
            copy_box(sm.sf[s] + 512, &p.x_exps, w.tok >> 7, kb >> 2, mbar);
          }
        }
        __syncwarp();
      }
      if (++s == kStages) s = 0, phase ^= 1;
    }
  }
  if (!ok && !half)  // copies in flight, the partner's too, land before either block ends
    for (uint32_t j = n > kStages ? n - kStages : 0; j < n; ++j)
      (void)mbar_wait(&sm.full[j % kStages], (j / kStages) & 1, x.wait_ns);
}

__device__ void mma_role(const GemmArgs& a, Smem& sm, const Ctx& x, uint32_t tmem, uint16_t both) {
  uint32_t n = 0, c = 0;           // blocks, chunks so far
  uint32_t s = 0, phase = 0;       // stage of block n
  SfSets sets;
  bool ok = true, ready = false;  // the stage of the next block was seen full
  const uint32_t bufs = a.n <= kTwoBufs ? 2 : 1, idesc0 = idesc_mx(2 * BM, a.n), sfs = sf_tiles(a.n);
  const uint64_t tile0 = desc_rows(smem_addr(sm.tile[0])), sf0 = desc_sf(smem_addr(sm.sf[0]));
  for (Walk w(a); ok && w.more(); w.next(a.n), ++c) {
    const uint32_t buf = c % bufs, d = tmem + buf * a.n;
    const uint32_t shift = 4 + ((uint32_t)(w.tok & 127) >> 5);
    uint32_t sfa = tmem + kSfAt + sets.at() * kSfCols;
    if (!(ok = wait_cluster_warp(x, &sm.acc_empty[buf], ((c / bufs) & 1) ^ 1))) break;
    tc_fence_after();
    for (int kb = w.k0; kb < w.k1; ++kb, ++n) {
      if (!__all_sync(0xffffffffu, ready) && !(ok = wait_cluster_warp(x, &sm.full[s], phase))) break;
      tc_fence_after();
      const bool sf = (kb & 3) == 0 || kb == w.lo;
      if (sf) {
        if (!(ok = sets.open<kStages, 2>(x, sm.empty, n))) break;
        sfa = tmem + kSfAt + sets.at() * kSfCols;
      }
      const uint64_t ds = sf0 + s * (kSfBytes / 16);
      const uint32_t idesc = with_sf_id(idesc0, kb & 3), sfb = sfa + shift;
      const uint64_t da = tile0 + s * (kStageBytes / 16), db = da + BM * 128 / 16;
      const bool end = s + 1 == kStages;
      ready = mbar_test_cluster(&sm.full[end ? 0 : s + 1], end ? phase ^ 1 : phase);
      if (one_lane()) {
        if (sf) {
          copy_sf(sfa, ds);
          copy_sf(sfa + 4, ds + 32);
          if (sfs > 1) copy_sf(sfa + 8, ds + 64);
        }
        umma_mx(d, da, db, idesc, sfa, sfb, kb != w.k0);
#pragma unroll
        for (int j = 1; j < 4; ++j) umma_mx(d, da + 2 * j, db + 2 * j, idesc, sfa, sfb, 1);
        // a commit holds the tensor cores up for 74 cycles (a block's products take 512): one for two stages
        if (n & 1) commit_both(&sm.empty[s >> 1], both);
        if (kb + 1 == w.k1) commit_both(&sm.acc_full[buf], both);
      }
      __syncwarp();
      s = end ? 0 : s + 1;
      phase ^= end;
    }
  }
  if (!ok && one_lane()) {  // products in flight end before the block does
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_addr(&sm.drain)) : "memory");
    (void)mbar_wait(&sm.drain, 0, x.wait_ns);
  }
}

__device__ void write_role(const GemmArgs& a, Smem& sm, const Ctx& x, uint32_t tmem, uint32_t half, uint32_t even) {
  constexpr int kPer = kMaxN / 2;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, per = a.n >> 1;
  const uint32_t quarter = warp & 3, c0 = (warp >> 2) * per, bufs = a.n <= kTwoBufs ? 2 : 1;
  float acc[kPer];
  uint32_t c = 0;
  for (Walk w(a); w.more(); w.next(a.n), ++c) {
    const uint32_t buf = c % bufs;
    if (!wait_warp(x, &sm.acc_full[buf], (c / bufs) & 1)) return;
    tc_fence_after();
    const uint32_t t = tmem + ((quarter * 32) << 16) + buf * a.n + c0;
    if (w.first()) {
#pragma unroll
      for (int i = 0; i < kPer; i += 16)
        if (i < per) tmem_ld16(t + i, acc + i);
      tmem_wait_ld(acc);
#pragma unroll
      for (int i = 16; i < kPer; i += 16) tmem_tie(acc + i);
    } else {
#pragma unroll
      for (int i = 0; i < kPer; i += 16)
        if (i < per) {
          float v[16];
          tmem_ld16(t + i, v);
          tmem_wait_ld(v);
#pragma unroll
          for (int j = 0; j < 16; ++j) acc[i + j] = __fadd_rn(acc[i + j], v[j]);
        }
    }
    tc_fence_before();
    __syncwarp();
    if (lane == 0) arrive_at(peer_addr(&sm.acc_empty[buf], even));
    if (!w.last()) continue;
    const int r = quarter * 32 + lane, row = w.row + BM * half + r;
    if (a.split > 1) {  // the part stays here until the cluster joins it; all copies and products of the pair are done
      float* part = reinterpret_cast<float*>(sm.tile[0]);
#pragma unroll
      for (int i = 0; i < kPer; ++i)
        if (i < per) part[(c0 + i) * BM + r] = acc[i];
    } else if (a.vec_y) {
      const int have = min(per, a.x.rows - w.tok - (int)c0) - (lane & 3), tok = w.tok + c0 + (lane & 3);
#pragma unroll
      for (int i = 0; i < kPer; i += 4)
        if (i < per) {
          const float4 v = quad(acc[i], acc[i + 1], acc[i + 2], acc[i + 3]);
          if (i < have) put4(a, tok + i, row & ~3, v);
        }
    } else if (row < a.w.rows) {
      const int have = min(per, a.x.rows - w.tok - (int)c0);
#pragma unroll
      for (int i = 0; i < kPer; ++i)
        if (i < have) put(a, w.tok + c0 + i, row, acc[i]);
    }
  }
}

__device__ void join(const GemmArgs& a, Smem& sm, uint32_t half) {
  const Walk w(a);
  const int share = (blockIdx.x >> 1) % a.split, row0 = w.row + BM * half;
  const int cols = min(a.n, a.x.rows - w.tok);
  constexpr int kAhead = 4;  // parts of so many elements under way together
  const int step = a.split * kThreads;
  for (int e0 = share * kThreads + threadIdx.x; e0 < cols * (BM / 4); e0 += kAhead * step) {
    float4 v[kAhead][kMaxSplit];
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
      if (e0 + i * step < cols * (BM / 4)) get_parts<kMaxSplit>(v[i], smem_addr(sm.tile[0]) + 16 * (e0 + i * step), half, 2, a.split);
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int e = e0 + i * step;
      if (e < cols * (BM / 4)) put4(a, w.tok + e / (BM / 4), row0 + e % (BM / 4) * 4, sum_parts<kMaxSplit>(v[i], a.split));
    }
  }
}

__global__ void __launch_bounds__(kThreads, 1) fp8_pairs_kernel(const __grid_constant__ PairArgs p) {
  const GemmArgs& a = p.g;
  extern __shared__ unsigned char smem_raw[];
  Smem& sm = *reinterpret_cast<Smem*>(smem_raw + ((1024u - (smem_addr(smem_raw) & 1023u)) & 1023u));
  const int warp = threadIdx.x >> 5;
  const uint32_t rank = cluster_rank(), half = rank & 1, even = rank & ~1u;
  if (warp == kCopyWarp && (threadIdx.x & 31) < 4)  // the four tensors' descriptors
    asm volatile("prefetch.tensormap [%0];" ::"l"(&p.w_codes + (threadIdx.x & 31)) : "memory");
  if (warp == kMmaWarp) {
    if ((threadIdx.x & 31) == 0) {
      for (int i = 0; i < kStages; ++i) mbar_init(&sm.full[i], 1);
      for (int i = 0; i < kStages / 2; ++i) mbar_init(&sm.empty[i], 1);
      for (int i = 0; i < 2; ++i) mbar_init(&sm.acc_full[i], 1), mbar_init(&sm.acc_empty[i], 16);
      mbar_init(&sm.drain, 1);
      sm.dead = 0;
      asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncwarp();
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&sm.tmem)), "r"(512)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    tc_fence_before();
  }
  __syncwarp();
  cluster_sync();  // both thread blocks' barriers and tensor memory are there
  tc_fence_after();
  step_trigger();
  const Ctx x{a.wait_ns, a.status, &sm.dead};
  const uint32_t tmem = sm.tmem;
  if (warp < 8) {
    step_wait();
    write_role(a, sm, x, tmem, half, even);
  } else if (warp == kCopyWarp) {
    copy_role(p, sm, x, half, even);
  } else if (!half) {
    mma_role(a, sm, x, tmem, (uint16_t)(3u << even));
  }
  __syncwarp();
  tc_fence_before();
  cluster_sync();  // every block gets here: all its waits are bounded
  if (warp == kMmaWarp) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
  }
  if (a.split > 1) {
    __syncwarp();
    join(a, sm, half);
    __syncwarp();
    cluster_sync();  // no block leaves while others read its part
  }
}

// A tensor [blocks][rows][`row` bytes], read in boxes of `box` rows.
cudaError_t tensor(CUtensorMap* map, CUtensorMapDataType type, int size, const void* p, int row, int64_t rows, int64_t blocks,
                   int box) {
  const cuuint64_t dims[3] = {(cuuint64_t)(row / size), (cuuint64_t)rows, (cuuint64_t)blocks};
  const cuuint64_t strides[2] = {(cuuint64_t)row, (cuuint64_t)(row * rows)};
  const cuuint32_t boxes[3] = {(cuuint32_t)(row / size), (cuuint32_t)box, 1};
  return make_tensor_map(map, type, 3, p, dims, strides, boxes);
}

cudaError_t launch(const GemmArgs& a, cudaStream_t st) {
  constexpr int kSmem = (int)sizeof(Smem) + 1024;
  static_assert(kSmem <= 227 * 1024, "shared memory of a block");
  static_assert(kMaxN * BM * 4 <= kStages * kStageBytes, "a part of a tile fits into the stages");
  static_assert(2 * kTwoBufs <= kSfAt && kMaxN <= kSfAt, "accumulators end before the scales");
  cudaError_t e = allow_smem<Smem>(fp8_pairs_kernel, kSmem);
  PairArgs p;
  p.g = a;
  const int blocks = a.x.blocks(), fours = (blocks + 3) / 4;
  for (const bool is_x : {false, true}) {
    const Fp8Mat& m = is_x ? a.x : a.w;
    if (e == cudaSuccess)
      e = tensor(is_x ? &p.x_codes : &p.w_codes, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, m.codes, 128, m.rows8(), blocks,
                 is_x ? a.n / 2 : BM);
    if (e == cudaSuccess)
      e = tensor(is_x ? &p.x_exps : &p.w_exps, CU_TENSOR_MAP_DATA_TYPE_UINT32, 4, m.exps, 512, m.tiles(), fours,
                 is_x ? sf_tiles(a.n) : 1);
  }
  if (e != cudaSuccess) return e;
  const int64_t tiles = (int64_t)((a.w.tiles() + 1) / 2) * ((a.x.rows + a.n - 1) / a.n);
  const int64_t pairs = a.split > 1 ? tiles * a.split : tiles < kPairs ? tiles : kPairs;
  return launch_step(fp8_pairs_kernel, dim3((unsigned)(2 * pairs)), kThreads, kSmem, 2 * a.split, st, p);
}

}  // namespace

cudaError_t make_tensor_map(CUtensorMap* map, CUtensorMapDataType type, int rank, const void* p, const cuuint64_t* dims,
                            const cuuint64_t* strides, const cuuint32_t* box) {
  typedef decltype(&cuTensorMapEncodeTiled) Encode;
  static const Encode encode = [] {
    void* f = nullptr;
    cudaDriverEntryPointQueryResult found;
    const cudaError_t e = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &found);
    return e == cudaSuccess && found == cudaDriverEntryPointSuccess ? reinterpret_cast<Encode>(f) : nullptr;
  }();
  if (!encode) return cudaErrorNotSupported;
  const cuuint32_t ones[3] = {1, 1, 1};
  const CUresult r = encode(map, type, rank, const_cast<void*>(p), dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
                            CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

cudaError_t max_clusters(fp8::Clusters* most) {
  constexpr int kDevices = 64, kMost = 8;
  static std::atomic<int> known[kDevices][kMost + 1];  // 1 + the answer; 0: not asked yet, or the question failed
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  most->of[0] = 0;
  most->of[1] = kSms;
  for (int size = 2; size <= kMost && e == cudaSuccess; ++size) {
    const int k = dev < kDevices ? known[dev][size].load(std::memory_order_relaxed) : 0;
    if (k) {
      most->of[size] = k - 1;
      continue;
    }
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = size;
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(size);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = sizeof(Smem) + 1024;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    e = allow_smem<Smem>(fp8_pairs_kernel, (int)cfg.dynamicSmemBytes);
    if (e == cudaSuccess) e = cudaOccupancyMaxActiveClusters(&most->of[size], fp8_pairs_kernel, &cfg);
    if (e == cudaSuccess && dev < kDevices) known[dev][size].store(most->of[size] + 1, std::memory_order_relaxed);
  }
  return e;
}

cudaError_t launch_fp8_pairs(const GemmArgs& in, cudaStream_t st) {
  GemmArgs a = in;
  Clusters most;
  const cudaError_t e = max_clusters(&most);
  if (e != cudaSuccess) return e;
  const Choice c = choose_pairs(a.w.rows, a.x.blocks(), a.x.rows, most);
  a.n = c.n;
  a.split = c.split;
  return launch(a, st);
}

}  // namespace awsrc
