// fp8_gemm.cu — y = x w^T for two matrices held in e4m3 codes with one
// power-of-two scale per row and 128 columns, on the fifth-generation tensor cores:
// the choice between two kernels, and the one for few rows of x.
//
// Mathematics: y[t][i] = sum_b 2^(ex[t][b] + ew[i][b]) sum_{k in b} cx[t][k] cw[i][k].
// The scales are powers of two, so the tensor cores apply them
// (kind::mxf8f6f4, scales of 8 exponent bits): one scale stands for four groups of
// 32 columns, the same byte for each of a block's four products.
//
// Few rows of x (up to 64: single tokens, drafts): the bytes of w bound it. A tile is R
// rows of w (tensor memory's lanes, up to 128 used) x N rows of x (columns), R such that
// every SM has the same share: one SM draws 50 GB/s, so the copy rate needs all of them.
//   Warp 8 copies: codes lie in memory as the tensor cores read them (rows of 128 bytes,
//     their 16-byte pieces exchanged by row), so a block's rows are one bulk copy, and a
//     ring of stages keeps the memory busy.
//   Up to 16 rows of x lie in shared memory before the products start, their codes copied
//     or, by warps 0-7, made here. Every thread block makes all rows' codes of its columns:
//     x 2048 x 11008 float32 took 6.9 us for one row, 8.4 for three, 17.6 for 16; with a
//     kernel for that in front 9.1, 9.5 and 9.6 (bf16 7.3, 9.7, 21.6 and 9.6 each; weights
//     from memory). Longer x, and 17 to 64 rows, come with w, block by block (made
//     here block by block, 40 rows took 29 us where both kernels took 17: each stage waited
//     for a copy, the codes and a fence).
//   Warp 10 puts the scales of the tile's rows of w in the order of its lanes. Warp 9
//     issues the products: 22 ns for each of a block's four and 167 ns for what a stage
//     costs all roles, so a stage holds two blocks. Warps 0-7 read the sums and write y.
// Few rows of w: a cluster shares a tile's columns and joins its parts, in their order,
// through shared memory.
//
// Measured with the quantising of x, in a captured run with weights from memory: one row x
// 2048 x 11008 float32 7.4 us (floor 3.4, w's bytes at the copy rate; out of the L2 5.9), 40
// x 3584 x 18944 bf16 17.4 us (floor 10.4). Left are what lies before the first product (2.3
// us; with a kernel in front 3.8, while the first stages of w arrive) and the results' way
// out (1 us).
//
// Every wait is bounded (wait_ns): one that runs out sets bit 2 of the fault word,
// stops the block's roles, waits (bounded) for its copies and products in flight
// and frees the tensor memory.
#include "fp8_codes.cuh"
#include "fp8_mma.cuh"
#include "internal.h"

namespace awsrc {

namespace {

using namespace fp8;

constexpr int kThreads = 352, kXWarps = 8, kCopyWarp = 8, kMmaWarp = 9, kScaleWarp = 10;
constexpr int kMaxSplit = kFewSplit;
// (row, block) pairs of x that a thread block quantises in the product's kernel at most; each takes
// 45 ns (bf16 60), a kernel for that in front and its end 2 to 2.5 us
constexpr int kOwnF32 = 56, kOwnBf16 = 32;

// Where x comes from: its codes with the blocks of w; all codes first; all rows first, quantised here.
enum Source { kCodes, kCodesFirst, kF32First, kBf16First };

template <int N, Source X>
struct Cfg {
  static constexpr bool kFirst = X != kCodes, kRaw = X == kF32First || X == kBf16First;
  static constexpr int kWBytes = BM * 128, kXAt = 2 * kWBytes;  // a stage holds two blocks: rows of w, then of x
  static constexpr int kStageBytes = kXAt + (kFirst ? 0 : 2 * N * 128);
  static constexpr int kStages = kFirst || N > 32 ? 4 : 5;
  static constexpr int kXBytes = kFirst ? 64 * 1024 : 0;  // codes of x that come first
  static constexpr int kXGroups = kFirst ? 18 : kStages;  // their scales, 512 bytes for 4 blocks; else of a stage
  static constexpr int kAccCols = 2 * N;                  // two accumulators
  static constexpr int kSfCols = 8;                       // a set of scales: 4 columns for w, 4 for x
  static constexpr int kCols = kAccCols + kSfSets * kSfCols;
  static constexpr int kTmem = kCols > 128 ? 256 : 128;
};

template <int N, Source X>
struct Smem {
  using C = Cfg<N, X>;
  uint8_t tile[C::kStages][C::kStageBytes];
  uint8_t x[C::kXBytes + 1024];  // a block's last rows of 16 may lie in the next one's place
  uint8_t sf_w[C::kStages][512], sf_raw[C::kStages][1024], sf_x[C::kXGroups][512];
  unsigned long long full[C::kStages], empty[C::kStages], raw_full[C::kStages], acc_full[2], acc_empty[2], x_full, drain;
  uint32_t tmem;
  int dead;
};

// Bytes of a block of x's codes: 8 or 16 rows.
__device__ __forceinline__ uint32_t x_block(const GemmArgs& a) { return a.x.rows8() * 128; }

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

// The walk that all roles take: tiles of this block, its share of their columns (whole
// stages but for the last) in chunks of blocks.
struct Walk {
  int tiles, chunk, step;
  int tile, lo, hi, k0, k1;
  __device__ explicit Walk(const GemmArgs& a) {
    tiles = (a.w.rows + a.n - 1) / a.n;
    const unsigned blocks = a.w.blocks(), split = a.split, rank = blockIdx.x % split;  // at most 2^17 blocks, 8 shares
    const unsigned twos = (blocks + 1) / 2;
    step = gridDim.x / split;
    tile = blockIdx.x / split;
    lo = 2 * (twos * rank / split);
    hi = min(blocks, 2 * (twos * (rank + 1) / split));
    chunk = a.y_f32 ? kChunkF32 : kChunkBf16;
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

// ------------------------------------------------------------------- copies
template <int N, Source X>
__device__ void copy_role(const GemmArgs& a, Smem<N, X>& sm, const Ctx& x) {
  using C = Cfg<N, X>;
  const int lane = threadIdx.x & 31;
  const int64_t w8 = a.w.rows8(), w_step = w8 * 128;
  const uint32_t xb = x_block(a);
  Walk w(a);
  const auto has_sf = [&](int kb) { return (kb & 3) == 0 || kb == w.lo; };
  // a stage begins: what its barriers count
  const auto expect = [&](int kb, uint32_t s) {
    const int row = w.tile * a.n, m = min(2, w.hi - kb);
    mbar_expect_tx(&sm.full[s], m * 128u * (uint32_t)min((int64_t)a.n, w8 - row) + (C::kFirst ? 0u : m * xb + (has_sf(kb) ? 512u : 0u)));
    // scales of the one or two tiles of 128 rows that this tile's rows lie in
    const uint32_t sf = has_sf(kb) ? 512u * (uint32_t)min(2, a.w.tiles() - (row >> 7)) : 0u;
    mbar_expect_tx(&sm.raw_full[s], sf);
    if (sf) bulk_g2s(sm.sf_raw[s], a.w.exps + ((int64_t)(kb >> 2) * a.w.tiles() + (row >> 7)) * 512, sf, &sm.raw_full[s]);
  };
  const auto copy_w = [&](int kb, uint32_t s, const uint8_t* rows) {
    bulk_g2s(sm.tile[s] + (kb & 1) * C::kWBytes, rows, 128u * (uint32_t)min((int64_t)a.n, w8 - w.tile * a.n), &sm.full[s]);
  };
  const auto copy_x = [&](int kb, uint32_t s) {
    bulk_g2s(sm.tile[s] + C::kXAt, a.x.codes + (int64_t)kb * xb, min(2, w.hi - kb) * xb, &sm.full[s]);
    if (has_sf(kb)) bulk_g2s(sm.sf_x[s], a.x.exps + (int64_t)(kb >> 2) * 512, 512, &sm.full[s]);
  };
  int ahead = 0;  // blocks of w on their way before x is ready
  if (a.early && a.stall < 0 && w.more()) {
    ahead = min(2 * C::kStages, w.hi - w.lo);
    if (lane < ahead) {
      if ((lane & 1) == 0) expect(w.lo + lane, lane >> 1);
      copy_w(w.lo + lane, lane >> 1, a.w.codes + (w.lo + lane) * w_step + w.tile * a.n * 128ll);
    }
    __syncwarp();
  }
  step_wait();
  if (X == kCodesFirst && w.more()) {
    if (lane == 0) {
      const int g0 = w.lo >> 2, groups = ((w.hi - 1) >> 2) - g0 + 1;
      mbar_expect_tx(&sm.x_full, (w.hi - w.lo) * xb + groups * 512u);
    }
    __syncwarp();
    for (int kb = w.lo + lane; kb < w.hi; kb += 32) {
      bulk_g2s(sm.x + (kb - w.lo) * xb, a.x.codes + (int64_t)kb * xb, xb, &sm.x_full);
      if (has_sf(kb)) bulk_g2s(sm.sf_x[(kb >> 2) - (w.lo >> 2)], a.x.exps + (int64_t)(kb >> 2) * 512, 512, &sm.x_full);
    }
    __syncwarp();
  }
  uint32_t n = 0, s = 0, phase = 1;  // stages so far; stage of block kb
  bool ok = true;
  for (; ok && w.more(); w.next()) {
    const uint8_t* rows = a.w.codes + w.k0 * w_step + w.tile * a.n * 128ll;
    for (int kb = w.k0; kb < w.k1; kb += 2, ++n, rows += 2 * w_step) {
      if (kb == (a.stall & ~1) || !wait_warp(x, &sm.empty[s], phase)) {
        ok = false;
        break;
      }
      if (one_lane()) {
        const bool begun = (int)(2 * n) < ahead;
        if (!begun) expect(kb, s);
        if (!C::kFirst) copy_x(kb, s);
        if (!begun) {
          copy_w(kb, s, rows);
          if (kb + 1 < w.k1) copy_w(kb + 1, s, rows + w_step);
        }
      }
      __syncwarp();
      if (++s == C::kStages) s = 0, phase ^= 1;
    }
  }
  if (!ok)  // copies in flight land before the block ends; where others did not come, the limit is time enough for all
    for (uint32_t j = n > C::kStages ? n - C::kStages : 0; j < n; ++j)
      if (!mbar_wait(&sm.full[j % C::kStages], (j / C::kStages) & 1, x.wait_ns)) break;
}

// --------------------------------------------------- scales of the rows of w
// The scale word of row r of the tile goes to lane r % 32, word r / 32.
template <int N, Source X>
__device__ void scale_role(const GemmArgs& a, Smem<N, X>& sm, const Ctx& x) {
  using C = Cfg<N, X>;
  const int lane = threadIdx.x & 31;
  uint32_t s = 0, phase = 0;
  for (Walk w(a); w.more(); w.next())
    for (int kb = w.k0; kb < w.k1; kb += 2) {
      if (!wait_warp(x, &sm.raw_full[s], phase)) return;
      if ((kb & 3) == 0 || kb == w.lo) {
        uint32_t v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int r = (w.tile * a.n & 127) + lane + 32 * i;
          v[i] = r < 256 ? *reinterpret_cast<const uint32_t*>(&sm.sf_raw[s][(r >> 7) * 512 + (r & 31) * 16 + ((r & 127) >> 5) * 4]) : 0u;
        }
        *reinterpret_cast<uint4*>(&sm.sf_w[s][lane * 16]) = make_uint4(v[0], v[1], v[2], v[3]);
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
      }
      if (lane == 0) mbar_arrive(&sm.full[s]);
      if (++s == C::kStages) s = 0, phase ^= 1;
    }
}

// --------------------------------------------------------------- codes of x
__device__ __forceinline__ void get4(const float* p, int have, bool vec, float* v) { vec ? load4<true>(p, have, v) : load4<false>(p, have, v); }
__device__ __forceinline__ void get4(const __nv_bfloat16* p, int have, bool vec, float* v) { vec ? load4<true>(p, have, v) : load4<false>(p, have, v); }

// All of this block's columns of all rows of x: (row, block) pairs over the warps, four in flight
// in each warp.
template <int N, Source X, typename T>
__device__ void quantize_role(const GemmArgs& a, Smem<N, X>& sm) {
  constexpr int kAhead = 4;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, M = a.x.rows, blocks = a.w.blocks();
  const uint32_t xb = x_block(a);
  const Walk w(a);
  const int pairs = w.more() ? (w.hi - w.lo) * M : 0;
  step_wait();
  for (int p0 = warp; p0 < pairs; p0 += kAhead * kXWarps) {
    float v[kAhead][4];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int p = p0 + i * kXWarps, kb = w.lo + p / M, r = p % M;
      if (p < pairs)
        get4(static_cast<const T*>(a.raw) + r * a.raw_stride + 128ll * kb + 4 * lane, a.x.cols - (128 * kb + 4 * lane), a.vec_raw, v[i]);
    }
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int p = p0 + i * kXWarps, kb = w.lo + p / M, r = p % M;
      if (p >= pairs) break;
      const Codes4 c = codes_of(v[i], a.x.cols - (128 * kb + 4 * lane));
      const int at = r * 128 + 16 * ((lane >> 2) ^ (r & 7)) + 4 * (lane & 3);
      const bool keep = kb % w.tiles == w.tile;  // each block's codes are left in x8 by one tile's thread block
      *reinterpret_cast<uint32_t*>(sm.x + (kb - w.lo) * xb + at) = c.codes;
      if (keep) *reinterpret_cast<uint32_t*>(a.x.codes + (int64_t)kb * xb + at) = c.codes;
      if (lane == 0) {
        sm.sf_x[(kb >> 2) - (w.lo >> 2)][r * 16 + (kb & 3)] = (uint8_t)c.biased;
        if (keep) {
          uint8_t* e = a.x.exps + (int64_t)(kb >> 2) * 512 + r * 16;
          e[kb & 3] = (uint8_t)c.biased;
          if (kb + 1 == blocks)
            for (int b = (kb & 3) + 1; b < 4; ++b) e[b] = 0;
        }
      }
    }
  }
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  __syncwarp();
  if (lane == 0) mbar_arrive(&sm.x_full);
}

// ----------------------------------------------------------------- products
template <int N, Source X>
__device__ void mma_role(const GemmArgs& a, Smem<N, X>& sm, const Ctx& x, uint32_t tmem) {
  using C = Cfg<N, X>;
  uint32_t n = 0, c = 0;      // stages, chunks so far
  uint32_t s = 0, phase = 0;  // stage of block kb
  SfSets sets;
  const uint32_t idesc0 = idesc_mx(BM, N), xb = x_block(a) / 16;
  const uint64_t tile0 = desc_rows(smem_addr(sm.tile[0])), x0 = desc_rows(smem_addr(sm.x));
  const uint64_t w_sf = desc_sf(smem_addr(sm.sf_w[0])), x_sf = desc_sf(smem_addr(sm.sf_x[0]));
  bool ok = true, ready = false;  // the next stage was seen full
  Walk w(a);
  if (C::kFirst && w.more()) ok = wait_warp(x, &sm.x_full, 0);
  for (; ok && w.more(); w.next(), ++c) {
    const uint32_t buf = c & 1, d = tmem + buf * N;
    uint32_t sfa = tmem + C::kAccCols + C::kSfCols * sets.at();
    if (!(ok = wait_warp(x, &sm.acc_empty[buf], ((c >> 1) & 1) ^ 1))) break;
    tc_fence_after();
    for (int kb = w.k0; kb < w.k1; kb += 2, ++n) {
      if (!__all_sync(0xffffffffu, ready) && !(ok = wait_warp(x, &sm.full[s], phase))) break;
      tc_fence_after();
      const bool sf = (kb & 3) == 0 || kb == w.lo;
      if (sf) {
        if (!(ok = sets.open<C::kStages, 1>(x, sm.empty, n))) break;
        sfa = tmem + C::kAccCols + C::kSfCols * sets.at();
      }
      const uint32_t id0 = with_sf_id(idesc0, kb & 3), id1 = with_sf_id(idesc0, (kb & 3) + 1);
      const uint64_t da = tile0 + s * (C::kStageBytes / 16), db = C::kFirst ? x0 + (kb - w.lo) * xb : da + C::kXAt / 16;
      const bool end = s + 1 == C::kStages, two = kb + 1 < w.k1;
      ready = mbar_test(&sm.full[end ? 0 : s + 1], end ? phase ^ 1 : phase);
      if (one_lane()) {
        if (sf) {
          copy_sf(sfa, w_sf + s * 32);
          copy_sf(sfa + 4, x_sf + (C::kFirst ? (kb >> 2) - (w.lo >> 2) : (int)s) * 32);
        }
        umma_mx(d, da, db, id0, sfa, sfa + 4, kb != w.k0);
#pragma unroll
        for (int j = 1; j < 4; ++j) umma_mx(d, da + 2 * j, db + 2 * j, id0, sfa, sfa + 4, 1);
        if (two) {
#pragma unroll
          for (int j = 0; j < 4; ++j) umma_mx(d, da + C::kWBytes / 16 + 2 * j, db + xb + 2 * j, id1, sfa, sfa + 4, 1);
        }
        umma_commit(&sm.empty[s]);
        if (kb + 2 >= w.k1) umma_commit(&sm.acc_full[buf]);
      }
      __syncwarp();
      s = end ? 0 : s + 1;
      phase ^= end;
    }
  }
  if (!ok && one_lane()) {  // products in flight end before the block does
    umma_commit(&sm.drain);
    (void)mbar_wait(&sm.drain, 0, x.wait_ns);
  }
}

// ------------------------------------------------------------------ results
template <int N, Source X>
__device__ void write_role(const GemmArgs& a, Smem<N, X>& sm, const Ctx& x, uint32_t tmem) {
  constexpr int kPer = N / 2;  // columns of a warp
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, r = 32 * (warp & 3) + lane, c0 = (warp >> 2) * kPer;
  float acc[kPer];
  uint32_t c = 0;
  for (Walk w(a); w.more(); w.next(), ++c) {
    const uint32_t buf = c & 1;
    if (!wait_warp(x, &sm.acc_full[buf], (c >> 1) & 1)) return;
    tc_fence_after();
    const uint32_t t = tmem + ((uint32_t)(r & ~31) << 16) + buf * N + c0;
    float v[kPer];
#pragma unroll
    for (int i = 0; i < kPer; i += 8) tmem_ld8(t + i, v + i);
    tmem_wait_ld8(v);
#pragma unroll
    for (int i = 8; i < kPer; i += 8) tmem_tie8(v + i);
    tc_fence_before();
    mbar_arrive(&sm.acc_empty[buf]);
#pragma unroll
    for (int i = 0; i < kPer; ++i) acc[i] = w.first() ? v[i] : __fadd_rn(acc[i], v[i]);
    if (!w.last()) continue;
    if (a.split > 1) {  // the part stays here until the cluster joins it; all copies and products of the block are done
      float* part = reinterpret_cast<float*>(sm.tile[0]);
#pragma unroll
      for (int i = 0; i < kPer; ++i) part[(c0 + i) * BM + r] = acc[i];
    } else if (a.vec_y) {
      const int row = w.tile * a.n + (r & ~3);  // a.n is a multiple of 8
#pragma unroll
      for (int i = 0; i < kPer; i += 4) {
        if (c0 + i >= a.x.rows) break;
        const float4 v = quad(acc[i], acc[i + 1], acc[i + 2], acc[i + 3]);
        if (c0 + i + (lane & 3) < a.x.rows && r < a.n) put4(a, c0 + i + (lane & 3), row, v);
      }
    } else if (const int row = w.tile * a.n + r; r < a.n && row < a.w.rows) {
#pragma unroll
      for (int i = 0; i < kPer; ++i)
        if (c0 + i < a.x.rows) put(a, c0 + i, row, acc[i]);
    }
  }
}

// The cluster's parts of a tile joined; each thread block joins its share of the elements.
template <int N, Source X>
__device__ void join(const GemmArgs& a, Smem<N, X>& sm) {
  constexpr int kAhead = 2;  // parts of so many elements under way together
  const int rank = blockIdx.x % a.split, row0 = blockIdx.x / a.split * a.n, per = a.n / 4, step = a.split * kThreads;
  for (int e0 = rank * kThreads + threadIdx.x; e0 < a.x.rows * per; e0 += kAhead * step) {
    float4 v[kAhead][kMaxSplit];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int e = e0 + i * step;
      if (e < a.x.rows * per) get_parts<kMaxSplit>(v[i], smem_addr(sm.tile[0]) + 4 * (e / per * BM + e % per * 4), 0, 1, a.split);
    }
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int e = e0 + i * step;
      if (e < a.x.rows * per) put4(a, e / per, row0 + e % per * 4, sum_parts<kMaxSplit>(v[i], a.split));
    }
  }
}

template <int N, Source X>
__global__ void __launch_bounds__(kThreads, 1) fp8_few_kernel(const __grid_constant__ GemmArgs a) {
  using C = Cfg<N, X>;
  extern __shared__ unsigned char smem_raw[];
  Smem<N, X>& sm = *reinterpret_cast<Smem<N, X>*>(smem_raw + ((1024u - (smem_addr(smem_raw) & 1023u)) & 1023u));
  const int warp = threadIdx.x >> 5;
  if (warp == kMmaWarp) {
    if ((threadIdx.x & 31) == 0) {
      for (int i = 0; i < C::kStages; ++i) {
        mbar_init(&sm.full[i], 2);
        mbar_init(&sm.empty[i], 1);
        mbar_init(&sm.raw_full[i], 1);
      }
      for (int i = 0; i < 2; ++i) mbar_init(&sm.acc_full[i], 1), mbar_init(&sm.acc_empty[i], 256);
      mbar_init(&sm.x_full, C::kRaw ? kXWarps : 1);
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
  step_trigger();
  const Ctx x{a.wait_ns, a.status, &sm.dead};
  const uint32_t tmem = sm.tmem;
  if (warp < kXWarps) {
    if constexpr (X == kF32First) quantize_role<N, X, float>(a, sm);
    if constexpr (X == kBf16First) quantize_role<N, X, __nv_bfloat16>(a, sm);
    step_wait();
    write_role(a, sm, x, tmem);
  } else if (warp == kCopyWarp) {
    copy_role(a, sm, x);
  } else if (warp == kMmaWarp) {
    mma_role(a, sm, x, tmem);
  } else {
    scale_role(a, sm, x);
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
    join(a, sm);
    __syncwarp();
    cluster_sync();  // no block leaves while others read its part
  }
}

cudaError_t choose(GemmArgs* a) {
  Clusters most;
  const cudaError_t e = max_clusters(&most);
  if (e != cudaSuccess) return e;
  const Choice c = choose_few(a->w.rows, a->w.blocks(), a->x.rows, most);
  a->n = c.n;
  a->split = c.split;
  return cudaSuccess;
}

template <int N, Source X>
cudaError_t launch(const GemmArgs& a, cudaStream_t st) {
  using C = Cfg<N, X>;
  constexpr int kSmem = (int)sizeof(Smem<N, X>) + 1024;
  static_assert(kSmem <= 227 * 1024, "shared memory of a block");
  static_assert(N * BM * 4 <= C::kStages * C::kStageBytes, "a part of a tile fits into the stages");
  const cudaError_t e = allow_smem<C>(fp8_few_kernel<N, X>, kSmem);
  if (e != cudaSuccess) return e;
  const int tiles = (a.w.rows + a.n - 1) / a.n;
  const int grid = a.split > 1 ? tiles * a.split : tiles < kSms ? tiles : kSms;
  static_assert(kChunkF32 % 2 == 0 && kChunkBf16 % 2 == 0, "chunks are whole stages");
  return launch_step(fp8_few_kernel<N, X>, dim3((unsigned)grid), kThreads, kSmem, a.split, st, a);
}

constexpr int kFewRows = 64, kFirstRows = 16;  // of x

// Blocks of columns that a thread block has at most.
int share_of(const GemmArgs& a) { return ((a.w.blocks() + 1) / 2 + a.split - 1) / a.split * 2; }

// Whether all codes of x of a thread block's columns fit beside the stages.
bool x_first(const GemmArgs& a) {
  return a.x.rows <= kFirstRows && share_of(a) * a.x.rows8() * 128 <= Cfg<16, kCodesFirst>::kXBytes;
}

}  // namespace

cudaError_t fp8_gemm_quantizes(const GemmArgs& in, bool bf16, bool* itself) {
  GemmArgs a = in;
  *itself = false;
  if (a.x.rows > kFirstRows) return cudaSuccess;
  const cudaError_t e = choose(&a);
  if (e == cudaSuccess) *itself = x_first(a) && a.x.rows * share_of(a) <= (bf16 ? kOwnBf16 : kOwnF32);
  return e;
}

cudaError_t launch_fp8_gemm(const GemmArgs& in, cudaStream_t st) {
  GemmArgs a = in;
  const uintptr_t size = a.y_f32 ? 4 : 2, raw_size = a.raw_bf16 ? 2 : 4;
  a.vec_y = (reinterpret_cast<uintptr_t>(a.y) | (uintptr_t)a.ys * size) % (4 * size) == 0;
  a.vec_raw = (reinterpret_cast<uintptr_t>(a.raw) | (uintptr_t)a.raw_stride * raw_size) % (4 * raw_size) == 0;
  cudaError_t e;
  if (a.x.rows > kFewRows) {
    e = launch_fp8_pairs(a, st);
  } else if ((e = choose(&a)) == cudaSuccess) {
    if (x_first(a))
      e = !a.raw ? launch<16, kCodesFirst>(a, st) : a.raw_bf16 ? launch<16, kBf16First>(a, st) : launch<16, kF32First>(a, st);
    else
      e = a.x.rows <= 16 ? launch<16, kCodes>(a, st) : a.x.rows <= 32 ? launch<32, kCodes>(a, st) : launch<64, kCodes>(a, st);
  }
  if (e != cudaSuccess) return e;
  note_launches(1);
  return cudaGetLastError();
}

}  // namespace awsrc
