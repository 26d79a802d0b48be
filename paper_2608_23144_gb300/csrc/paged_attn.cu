// paged_attn.cu — attention of a few query rows per kv head over the paged 8-bit
// cache: decode steps, drafts, and every case the tensor-memory kernel does not
// take.
//
// Mathematics, per kv head with scores in base 2: x_j = (q . k_j) 2^(ek_j)
// sm_scale log2(e) + ev_j, where 2^ek, 2^ev are the block scales of the codes.
// With m = max x, p_j = 2^(x_j - m + 15): O = sum p_j c_j over the value codes
// c_j and l = sum p_j 2^-ev_j give out = O / l and lse = (m - 15 + log2 l) ln 2.
// Putting 2^ev into the exponent leaves the codes to the tensor cores as they
// are (exact in binary16) and keeps p at most 2^15.
//
// Rows are query tokens x the query heads that share a kv head. Both products
// run transposed, tokens (or dims) as the 16 MMA rows and 8 query rows as the
// columns, so that a decode step of up to 8 heads per kv head wastes nothing.
// F32 splits q (scaled by a power of two per row) and p into two binary16 terms;
// the second term costs one more MMA on the same widened codes. (8-bit warp-level
// MMAs, which would take the codes as they are, run as conversions and 16-bit
// products here: 44 instead of 26 million instructions for the same batch.)
//
// Bound by the cache's bytes when rows are few. A block is 64 tokens; its keys
// and values come to shared memory by bulk copies (8 to 16 KB pieces, the cache's
// byte order being what the fragments want), one or two ahead of the products, so
// that what is in flight does not cost registers: loaded straight into registers,
// two blocks ahead made 57 KB of unrolled code whose cold fetch alone was 20 us of
// a single token's step. Lanes read 4-byte words without bank conflicts (keys:
// two-way). Fragment slots of lane (g, t): dims 16 i + 4 t + {0..3} in step i of
// q . k, tokens 16 s + 4 t + {0..3} in step s of p . V; score row tile s has token
// 16 s + 4 (g / 2) + g % 2 in row g and two further in row 8 + g.
//
// Decode (one row tile): four rings, each with every fourth block of a segment and
// two warps to halve it. Many rows: four warps hold 16 rows each and share one
// ring. Two thread blocks per SM, so that one's starts and ends of segments (a
// third of the time of 64 ragged sequences) pass under the other's products.
//
// Work: the (sequence, row tile, kv head, 64-token block) units of the batch in
// this order are dealt out in equal contiguous shares to the thread blocks,
// whatever the lengths. A tile that several blocks share is joined in block order
// from partial results in the workspace, by its last block to arrive or by a
// second launch; nothing waits.
//
// Measured: 64 ragged decode steps on contexts up to 8192 (28 heads, 4 kv heads,
// bf16) in 64 us, 5.3 TB/s of the cache; one on 131k tokens (40 heads, 8 kv heads,
// float32) in 54 us, 5.0 TB/s. In the loop the copies keep up with the memory;
// what is lost are the starts of blocks and the ends of segments (a tenth each) and,
// in float32, the second terms' products. Many float32 rows are bound by the
// warp-level MMAs, whose rate is a third of the fifth-generation cores': four
// prompts of up to 4096 tokens (28 heads, 4 kv heads) in 1.77 ms, 142 TFLOP/s.
//
// Rounding: q (bf16: exact; float32: 22 bits; either to 2^-25 under a largest element
// of 2^14), p (11 bits, float32: 22; either to 2^-25 under a largest p of 2^15; l takes
// it unrounded) and the widened codes (exact) to binary16; scores, m, l, O and the
// joins in binary32; out once. An MMA cuts its binary32 sums off instead of rounding
// them, so q's second terms have sums of their own, and a float32 weight gets its 2^15
// after the power, whose argument near zero keeps its last bits: together 8.5e-7 ->
// 4e-7 of the result for a token on 516 (4e-7 to 6e-7 over inputs).
#include "internal.h"
#include "kv_paged.cuh"
#include "tc05.cuh"

namespace awsrc {

namespace {

using namespace tc05;

constexpr int kUnit = 64;         // tokens per unit
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kPBits = 15.0f, kPMax = 32768.0f;  // p is at most 2^15
constexpr int kMaxParts = 8;      // parts of a tile that its last block joins

__device__ __forceinline__ void mma(float* c, const uint32_t* a, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// Transposes an 8 x 8 tile of binary16 held two columns per lane.
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
  return r;
}

__device__ __forceinline__ uint32_t half2_bits(float a, float b) {
  const __half2 h = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ float2 half2_floats(uint32_t v) { return __half22float2(*reinterpret_cast<const __half2*>(&v)); }

template <typename T>
__device__ __forceinline__ void load4(const T* p, bool vec, float* x);
template <>
__device__ __forceinline__ void load4(const float* p, bool vec, float* x) {
  if (vec) {
    const float4 v = *reinterpret_cast<const float4*>(p);
    x[0] = v.x, x[1] = v.y, x[2] = v.z, x[3] = v.w;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = p[i];
  }
}
template <>
__device__ __forceinline__ void load4(const __nv_bfloat16* p, bool vec, float* x) {
  if (vec) {
    const uint2 v = *reinterpret_cast<const uint2*>(p);
    x[0] = __uint_as_float(v.x << 16), x[1] = __uint_as_float(v.x & 0xFFFF0000u);
    x[2] = __uint_as_float(v.y << 16), x[3] = __uint_as_float(v.y & 0xFFFF0000u);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = __bfloat162float(p[i]);
  }
}

template <int NT, int WR>
struct Shape {
  static constexpr int kRowsPerWarp = 8 * NT;
  static constexpr int kRows = kRowsPerWarp * WR;  // query rows of a tile
  static constexpr int kTokWarps = 4 / WR;         // token groups: rings of blocks
  // warps that share a group's blocks, 64 / kH tokens each: two for decode steps,
  // whose few registers leave room for 16 warps on an SM
  static constexpr int kH = NT == 1 && WR == 1 ? 2 : 1;
  static constexpr int kWarps = 4 * kH, kThreads = 32 * kWarps;
  static constexpr int kParts = kTokWarps * kH;    // partial results of a row in the block
  // A segment's start and end, in blocks. Without them shares of several short
  // segments end late: 70 -> 66 us for 64 ragged decode steps (12; 8: 67, 16: 66),
  // 2.39 -> 1.69 ms for four float32 prompts (3; 2: 1.75, 5: 1.73).
  static constexpr int over(int dim) { return WR == 1 ? 12 : dim == 64 ? 2 : 3; }
  // thread blocks per SM: more where 64-dim heads leave registers for them
  static constexpr int blocks(int dim) { return dim == 64 && WR == 4 ? 4 : 2; }
};

template <int D>
struct RowStride { static constexpr int value = D + 4; };  // floats of a row in shared memory

__device__ __forceinline__ float inv_of(float l) { return l == 0.0f ? 0.0f : __frcp_rn(l); }

// Dims d .. d + 3 of row r of a finished tile: o / l by `inv`, and its lse.
template <typename T>
__device__ __forceinline__ void write4(const AttnArgs& a, const RowMap& map, int first, int r, int h, int d, const float4& o,
                                       float m, float l, float inv) {
  int tok, head;
  map.at(r, &tok, &head);
  tok += first;
  head += h * a.c.group;
  T* p = static_cast<T*>(a.out.p) + (int64_t)tok * a.out.ts + (int64_t)head * a.out.hs + d;
  const float v[4] = {__fmul_rn(o.x, inv), __fmul_rn(o.y, inv), __fmul_rn(o.z, inv), __fmul_rn(o.w, inv)};
  if constexpr (sizeof(T) == 2) {
    const __nv_bfloat162 b0 = __floats2bfloat162_rn(v[0], v[1]), b1 = __floats2bfloat162_rn(v[2], v[3]);
    if (a.vec_out) {
      *reinterpret_cast<uint2*>(p) = make_uint2(*reinterpret_cast<const uint32_t*>(&b0), *reinterpret_cast<const uint32_t*>(&b1));
    } else {
      p[0] = b0.x, p[1] = b0.y, p[2] = b1.x, p[3] = b1.y;
    }
  } else if (a.vec_out) {
    *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) p[i] = v[i];
  }
  if (d == 0 && a.lse) a.lse[(int64_t)tok * a.c.n_heads + head] = l == 0.0f ? -INFINITY : (m - kPBits + log2f(l)) * kLn2;
}

__device__ __forceinline__ float4 fma4(const float4& a, float f, const float4& c) {
  return make_float4(__fmaf_rn(a.x, f, c.x), __fmaf_rn(a.y, f, c.y), __fmaf_rn(a.z, f, c.z), __fmaf_rn(a.w, f, c.w));
}

// Shared memory: a ring of key and value blocks per token group. At a segment's
// end the warps' results lie over the values, while the next segment's first keys
// are on their way.
template <int D, int NT, int WR>
struct RowsSmem {
  using S = Shape<NT, WR>;
  static constexpr int kG = S::kTokWarps;                            // token groups
  static constexpr int NK = WR == 1 ? 2 : 3, NV = WR == 1 ? (D == 64 ? 2 : 1) : 3;
  using Walk = UnitWalk<S::kRows, kUnit, S::kWarps, S::over(D)>;
  uint8_t k[kG][NK][kUnit * D];
  union {
    uint8_t v[kG][NV][kUnit * D];
    struct {
      float o[S::kParts][S::kRows][RowStride<D>::value], m[S::kParts][S::kRows], l[S::kParts][S::kRows];
      float f[S::kParts][S::kRows];                             // a part's weight
      float mx[S::kRows], ls[S::kRows], inv[S::kRows];          // the row's m, l and 1 / l
    } out;
  };
  unsigned long long k_full[kG][NK], k_empty[kG][NK], v_full[kG][NV], v_empty[kG][NV];
  Walk walk;
  SegRec rec[2];
  int dead, last;
};

// What lanes 0 .. 3 know about the 16-token groups of a block: tokens in it (0
// for a page that cannot be right), its page and exponents.
struct Place {
  int pg, have, ek, ev;
};

// SMALL: pages of 16 tokens. A case of its own, since its copies cost the others
// 1 to 3 us of a decode step in registers.
template <typename T, int D, int NT, int WR, bool SMALL>
__global__ void __launch_bounds__(Shape<NT, WR>::kThreads, Shape<NT, WR>::blocks(D)) paged_rows_kernel(const __grid_constant__ AttnArgs a) {
  using S = Shape<NT, WR>;
  using Mem = RowsSmem<D, NT, WR>;
  constexpr int kI = D / 16;           // runs of 16 dims, and row tiles of p . V
  constexpr bool kSplit = sizeof(T) == 4;
  constexpr int kTerms = kSplit ? 2 : 1;
  extern __shared__ __align__(128) unsigned char smem_raw[];
  Mem& sm = *reinterpret_cast<Mem*>(smem_raw);
  const KvArgs& c = a.c;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int g = lane >> 2, t4 = lane & 3;
  constexpr int kH = S::kH, kT = 4 / kH;  // 16-token groups of a block per warp
  const int half = warp % kH, wr = warp / kH % WR, wt = warp / kH / WR;
  const bool feeds = wr == 0 && half == 0;  // the warp that copies for its token group
  const int log_pe = min(c.log_page, 6);  // tokens of a page within a block

  wait_for_previous();
  let_next_start();
  {
    typename Mem::Walk w;
    const bool any = w.start(a);
    if (a.shared && threadIdx.x == 0) a.shared[blockIdx.x] = SharedTile{};
    if (!any) return;
    if (threadIdx.x == 0) {
      sm.walk = w;
      Mem::Walk::next(&sm.walk, a, &sm.rec[0]);
    }
  }
  if (threadIdx.x == 0) {
    for (int i = 0; i < Mem::kG; ++i) {
      for (int j = 0; j < Mem::NK; ++j) mbar_init(&sm.k_full[i][j], SMALL ? 32 : 1), mbar_init(&sm.k_empty[i][j], WR * kH);
      for (int j = 0; j < Mem::NV; ++j) mbar_init(&sm.v_full[i][j], 1), mbar_init(&sm.v_empty[i][j], WR * kH);
    }
    sm.dead = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncthreads();
  // Bounded; once one has given up, all return at once and the results are void.
  auto wait = [&](unsigned long long* mb, uint32_t parity) {
    if (mbar_try_wait(mb, parity)) return true;
    const uint64_t t0 = globaltimer();
    while (!mbar_try_wait(mb, parity)) {
      if (*(volatile int*)&sm.dead) return false;
      if (globaltimer() - t0 > a.wait_ns) {
        *(volatile int*)&sm.dead = 1;
        atomicOr(c.status, kFaultTimeout);
        return false;
      }
    }
    return true;
  };

  uint32_t nk = 0, nv = 0;  // blocks of this group so far: issued by its first warp, waited for by all
  uint32_t ik = 0, iv = 0;
  auto find = [&](const SegRec& sg, int blk) {  // lanes 0 .. 3
    Place p{0, 0, 0, 0};
    const int j = blk * kUnit + 16 * (lane & 3);
    if (lane < 4 && blk < sg.blk1 && j < sg.kv) {
      const int pg = c.table[(int64_t)sg.b * c.table_stride + (j >> c.log_page)];
      if (pg >= 0 && pg < c.n_pages) {
        p.pg = pg;
        p.have = min(16, sg.kv - j);
        p.ek = __ldcg(c.k_exp + (int64_t)pg * c.kv_heads + sg.h);
        p.ev = __ldcg(c.v_exp + (int64_t)pg * c.kv_heads + sg.h);
      } else {
        atomicOr(c.status, kFaultBatch);
      }
    }
    return p;
  };
  // The copies of a block's keys or values by the group's feeding warp, to
  // [D / 16][64][16] and [4][D][16] whatever the page: values are in one piece
  // per page (half a page of 128), keys in one per page and 16 dims, or in one
  // where a page is a block.
  auto copy = [&](const Place& p, int h, int blk, bool keys) {
    const uint32_t n = keys ? ik++ : iv++;
    const int st = keys ? n % Mem::NK : n % Mem::NV;
    unsigned long long* full = keys ? &sm.k_full[wt][st] : &sm.v_full[wt][st];
    const bool ok = wait(keys ? &sm.k_empty[wt][st] : &sm.v_empty[wt][st], ((n / (keys ? Mem::NK : Mem::NV)) & 1) ^ 1);
    // nothing is copied into a stage that was not given back, or by the limit's test
    if (!__all_sync(0xffffffffu, ok) || (a.stall >= 0 && (int)n >= a.stall)) return;
    uint8_t* dst = keys ? sm.k[wt][st] : sm.v[wt][st];
    const uint8_t* src = (keys ? c.k : c.v) + (int64_t)h * (D << c.log_page);
    const int64_t page_bytes = (int64_t)c.kv_heads * (D << c.log_page);
    const int pe = 1 << log_pe, off = c.log_page > 6 ? (blk & 1) * kUnit : 0;  // tokens of a page in the block, first one
    const int pages = kUnit >> log_pe;
    // lane i < 4 holds group i; the first group of a page stands for it
    const bool first = lane < 4 && ((16 * lane) & (pe - 1)) == 0 && p.have > 0;
    const uint32_t got = __ballot_sync(0xffffffffu, first);
    if (SMALL && keys) {
#pragma unroll
      for (int j = 0; j < 2; ++j) {  // a page's run per half warp
        const int gi = 2 * j + (lane >> 4), pg = __shfl_sync(0xffffffffu, p.pg, gi);
        const uint8_t* from = src + pg * page_bytes + 16 * (lane & 15);
        if ((got >> gi) & 1) {
#pragma unroll
          for (int run = 0; run < kI; ++run) copy16(dst + (run * kUnit + 32 * j + lane) * 16, from + 256 * run);
        }
      }
      copies_arrive(full);
      return;
    }
    if (lane == 0) mbar_expect_tx(full, __popc(got) * D * pe);
    __syncwarp();
    const bool runs = keys && c.log_page != 6;
    const int pieces = runs ? pages * kI : pages;  // at most 32
    const int pgi = runs ? lane % pages : lane, run = runs ? lane / pages : 0, gi = (pgi << log_pe) >> 4;
    const int pg = __shfl_sync(0xffffffffu, p.pg, gi & 3);
    if (lane < pieces && ((got >> gi) & 1)) {
      const uint8_t* from = src + pg * page_bytes + (runs ? ((run << c.log_page) + off) * 16 : off * D);
      bulk_g2s(dst + (runs ? (run * kUnit + pgi * pe) * 16 : pgi * pe * D), from, runs ? pe * 16 : pe * D, full);
    }
  };

  // A segment's first blocks: their places, and their keys on their way.
  Place cur, nx[Mem::NK - 1];
  auto begin = [&](const SegRec& sg) {
    const int b0 = sg.blk0 + wt;
    cur = find(sg, b0);
#pragma unroll
    for (int i = 0; i < Mem::NK - 1; ++i) nx[i] = find(sg, b0 + (i + 1) * S::kTokWarps);
    if (feeds) {
      if (b0 < sg.blk1) copy(cur, sg.h, b0, true);
#pragma unroll
      for (int i = 0; i < Mem::NK - 1; ++i)
        if (b0 + (i + 1) * S::kTokWarps < sg.blk1) copy(nx[i], sg.h, b0 + (i + 1) * S::kTokWarps, true);
    }
  };
  if (sm.rec[0].b >= 0) begin(sm.rec[0]);
  for (int turn = 0; sm.rec[turn].b >= 0; turn ^= 1) {
    const SegRec& sg = sm.rec[turn];
    const int h = sg.h, rows = sg.rows, row0 = sg.row0, blk1 = sg.blk1, b0 = sg.blk0 + wt;
    if (threadIdx.x == 0) Mem::Walk::next(&sm.walk, a, &sm.rec[turn ^ 1]);
    if (feeds) {
      if (b0 < blk1) copy(cur, h, b0, false);
#pragma unroll
      for (int i = 0; i + 1 < Mem::NV; ++i)
        if (b0 + (i + 1) * S::kTokWarps < blk1) copy(nx[i], h, b0 + (i + 1) * S::kTokWarps, false);
    }

    // ---- query fragments: row wr kRowsPerWarp + 8 nt + g; a row past the last repeats it
    uint32_t qf[NT][kTerms][2 * kI];
    float rm[NT][2];     // score multiplier of rows 2 t4, 2 t4 + 1
    int lim[NT][2];      // last token these rows see
    int lim_min = INT32_MAX;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int r = wr * S::kRowsPerWarp + 8 * nt + g;
      const bool have = r < rows;
      const int row = row0 + min(r, rows - 1), tok = row / c.group;
      float x[4 * kI];
      const T* p = static_cast<const T*>(a.q.p) + (int64_t)(sg.first + tok) * a.q.ts +
                   (int64_t)(h * c.group + row - tok * c.group) * a.q.hs + 4 * t4;
#pragma unroll
      for (int i = 0; i < kI; ++i) load4(p + 16 * i, a.vec, x + 4 * i);
      float amax = 0.0f;
#pragma unroll
      for (int i = 0; i < 4 * kI; ++i) amax = fmax_nan(amax, fabsf(x[i]));
      amax = fmax_nan(amax, __shfl_xor_sync(0xffffffffu, amax, 1));
      amax = fmax_nan(amax, __shfl_xor_sync(0xffffffffu, amax, 2));
      // the row times 2^up has its largest element in [2^14, 2^15)
      const int ex = (int)(__float_as_uint(amax) >> 23) - 127;
      const int up = min(max(14 - ex, -120), 100);
      const float f = pow2f(up);
      const float mul = amax < INFINITY ? a.score_mul * pow2f(-up) : __int_as_float(0x7FC00000);
#pragma unroll
      for (int i = 0; i < 2 * kI; ++i) {
        const float y0 = __fmul_rn(x[2 * i], f), y1 = __fmul_rn(x[2 * i + 1], f);
        qf[nt][0][i] = half2_bits(y0, y1);
        if constexpr (kSplit) {
          const float2 hi = half2_floats(qf[nt][0][i]);
          qf[nt][1][i] = half2_bits(__fsub_rn(y0, hi.x), __fsub_rn(y1, hi.y));
        }
      }
      const int see = a.causal ? sg.kv - sg.n + tok : sg.kv - 1;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        rm[nt][i] = __shfl_sync(0xffffffffu, mul, 4 * (2 * t4 + i));
        lim[nt][i] = __shfl_sync(0xffffffffu, have ? see : -1, 4 * (2 * t4 + i));
      }
      int lo = have ? see : INT32_MAX;
#pragma unroll
      for (int o = 4; o < 32; o <<= 1) lo = min(lo, __shfl_xor_sync(0xffffffffu, lo, o));
      lim_min = min(lim_min, lo);
    }

    float o[NT][kI][4], m[NT][2], l[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
      for (int i = 0; i < 2; ++i) m[nt][i] = -INFINITY, l[nt][i] = 0.0f;
#pragma unroll
      for (int dt = 0; dt < kI; ++dt)
#pragma unroll
        for (int i = 0; i < 4; ++i) o[nt][dt][i] = 0.0f;
    }

    for (int blk = b0; blk < blk1; blk += S::kTokWarps) {
      const float nan = __int_as_float(0x7FC00000);
      const Place far = find(sg, blk + Mem::NK * S::kTokWarps);
      // some row is hidden from some token, or a group is short or marked
      const bool odd = cur.have < 16 || cur.ek == kExpNan || cur.ev == kExpNan;
      const bool masked = blk * kUnit + kUnit - 1 > lim_min || __any_sync(0xffffffffu, lane < 4 && odd);

      // ---- scores
      const int ks = nk % Mem::NK;
      wait(&sm.k_full[wt][ks], (nk / Mem::NK) & 1);
      ++nk;
      float x[NT][kT][4], xl[NT][kT][4];  // of q's first and second terms
      const uint8_t* kb = sm.k[wt][ks] + (4 * (g >> 1) + (g & 1)) * 16 + 4 * t4;
#pragma unroll
      for (int i = 0; i < kT; ++i)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int j = 0; j < 4; ++j) x[nt][i][j] = 0.0f, xl[nt][i][j] = 0.0f;
      const uint8_t* kp = kb + kT * half * 256;  // row tile i: 16 rows of 16 bytes further
      auto key = [&](int i, int run, int row) {
        return *reinterpret_cast<const uint32_t*>(kp + i * 256 + run * (kUnit * 16) + row * 16);
      };
      // products that follow one another go to different accumulators
#pragma unroll
      for (int j = 0; j < kI; ++j) {
        uint32_t fr[kT][4];
#pragma unroll
        for (int i = 0; i < kT; ++i) {
          widen4(key(i, j, 0), fr[i][0], fr[i][2]);
          widen4(key(i, j, 2), fr[i][1], fr[i][3]);
        }
#pragma unroll
        for (int q = kTerms - 1; q >= 0; --q)
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int i = 0; i < kT; ++i) mma(q == 0 ? x[nt][i] : xl[nt][i], fr[i], qf[nt][q][2 * j], qf[nt][q][2 * j + 1]);
      }
      if constexpr (kSplit) {
#pragma unroll
        for (int i = 0; i < kT; ++i)
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int j = 0; j < 4; ++j) x[nt][i][j] = __fadd_rn(x[nt][i][j], xl[nt][i][j]);
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&sm.k_empty[wt][ks]);
      if (feeds && blk + Mem::NK * S::kTokWarps < blk1) copy(far, h, blk + Mem::NK * S::kTokWarps, true);

      // ---- softmax weights
      uint32_t pf[NT][kTerms][2 * kT];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        float mx[2] = {-INFINITY, -INFINITY}, out[2] = {1.0f, 1.0f};
#pragma unroll
        for (int i = 0; i < kT; ++i) {
          const int gi = kT * half + i;
          const int ek = __shfl_sync(0xffffffffu, cur.ek, gi), ev = __shfl_sync(0xffffffffu, cur.ev, gi);
          const int have = __shfl_sync(0xffffffffu, cur.have, gi);
          const float sk = pow2f(ek), ef = ek == kExpNan ? nan : (ev == kExpNan ? 0.0f : (float)ev);
          const int j0 = blk * kUnit + 16 * gi + 4 * (g >> 1) + (g & 1);
          const int end = blk * kUnit + 16 * gi + have;
#pragma unroll
          for (int q = 0; q < 2; ++q) {
            const float k = __fmul_rn(rm[nt][q], sk);
#pragma unroll
            for (int hf = 0; hf < 2; ++hf) {
              x[nt][i][2 * hf + q] = __fmaf_rn(x[nt][i][2 * hf + q], k, ef);
            }
          }
          if (masked) {
#pragma unroll
            for (int q = 0; q < 2; ++q)
#pragma unroll
              for (int hf = 0; hf < 2; ++hf)
                if (j0 + 2 * hf >= end || j0 + 2 * hf > lim[nt][q]) x[nt][i][2 * hf + q] = -INFINITY;
            // a row that sees marked values: O is NaN, the scores and l are what they are
            if (ev == kExpNan) {
#pragma unroll
              for (int q = 0; q < 2; ++q)
                if (blk * kUnit + 16 * gi <= lim[nt][q]) out[q] = nan;
            }
          }
#pragma unroll
          for (int q = 0; q < 2; ++q) mx[q] = fmaxf(mx[q], fmaxf(x[nt][i][q], x[nt][i][2 + q]));
        }
        float base[2], al[2];
#pragma unroll
        for (int q = 0; q < 2; ++q) {
#pragma unroll
          for (int of = 4; of < 32; of <<= 1) mx[q] = fmaxf(mx[q], __shfl_xor_sync(0xffffffffu, mx[q], of));
          const float mn = fmaxf(m[nt][q], mx[q]);
          const float bs = mn == -INFINITY ? 0.0f : mn;
          al[q] = ex2(__fsub_rn(m[nt][q], bs));
          m[nt][q] = mn;
          base[q] = kSplit ? bs : __fsub_rn(bs, kPBits);
          l[nt][q] = __fmul_rn(l[nt][q], al[q]);
          al[q] = __fmul_rn(al[q], out[q]);
        }
        if (__any_sync(0xffffffffu, al[0] != 1.0f || al[1] != 1.0f)) {  // a maximum moved
#pragma unroll
          for (int dt = 0; dt < kI; ++dt)
#pragma unroll
            for (int q = 0; q < 4; ++q) o[nt][dt][q] = __fmul_rn(o[nt][dt][q], al[q & 1]);
        }
#pragma unroll
        for (int i = 0; i < kT; ++i) {
          const int ev = __shfl_sync(0xffffffffu, cur.ev, kT * half + i);
          const float un = pow2f(ev == kExpNan ? 0 : -ev);
#pragma unroll
          for (int hf = 0; hf < 2; ++hf) {
            float p0 = ex2(__fsub_rn(x[nt][i][2 * hf], base[0])), p1 = ex2(__fsub_rn(x[nt][i][2 * hf + 1], base[1]));
            if constexpr (kSplit) p0 = __fmul_rn(p0, kPMax), p1 = __fmul_rn(p1, kPMax);
            l[nt][0] = __fmaf_rn(p0, un, l[nt][0]);
            l[nt][1] = __fmaf_rn(p1, un, l[nt][1]);
            const uint32_t hi = half2_bits(p0, p1);
            pf[nt][0][2 * i + hf] = transpose8(hi);
            if constexpr (kSplit) {
              const float2 b = half2_floats(hi);
              pf[nt][1][2 * i + hf] = transpose8(half2_bits(__fsub_rn(p0, b.x), __fsub_rn(p1, b.y)));
            }
          }
        }
      }

      // ---- O^T += V^T P^T: row tiles of 16 dims, 4 steps of 16 tokens. Rows that
      // hold no token may hold any bytes, e4m3's NaN among them.
      const int vs = nv % Mem::NV;
      wait(&sm.v_full[wt][vs], (nv / Mem::NV) & 1);
      ++nv;
      if (masked && __any_sync(0xffffffffu, lane < 4 && cur.have < 16)) {
#pragma unroll 1
        for (int i = 0; i < kT; ++i) {
          const uint32_t keep = first_bytes(__shfl_sync(0xffffffffu, cur.have, kT * half + i) - 4 * t4);
#pragma unroll 1
          for (int d = g; d < D; d += 8)  // warps that share the ring all do it, to the same effect
            *reinterpret_cast<uint32_t*>(sm.v[wt][vs] + ((kT * half + i) * D + d) * 16 + 4 * t4) &= keep;
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");  // a copy overwrites it later
        __syncwarp();
      }
      const uint8_t* vb = sm.v[wt][vs] + g * 16 + 4 * t4;
      auto value = [&](int i, int dim) { return *reinterpret_cast<const uint32_t*>(vb + ((kT * half + i) * D + dim) * 16); };
#pragma unroll
      for (int i = 0; i < kT; ++i)
#pragma unroll
        for (int dt = 0; dt < kI; dt += 4) {
          uint32_t fr[4][4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            widen4(value(i, 16 * (dt + e)), fr[e][0], fr[e][2]);
            widen4(value(i, 16 * (dt + e) + 8), fr[e][1], fr[e][3]);
          }
#pragma unroll
          for (int q = kTerms - 1; q >= 0; --q)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
              for (int e = 0; e < 4; ++e) mma(o[nt][dt + e], fr[e], pf[nt][q][2 * i], pf[nt][q][2 * i + 1]);
        }
      __syncwarp();
      if (lane == 0) mbar_arrive(&sm.v_empty[wt][vs]);
      if (feeds && blk + Mem::NV * S::kTokWarps < blk1)
        copy(Mem::NV == Mem::NK ? far : nx[Mem::NV - 1], h, blk + Mem::NV * S::kTokWarps, false);
      cur = nx[0];
#pragma unroll
      for (int i = 0; i + 1 < Mem::NK - 1; ++i) nx[i] = nx[i + 1];
      nx[Mem::NK - 2] = far;
    }

    // ---- the warps' results to shared memory, over the values; the next
    // segment's first keys meanwhile
    __syncthreads();
    if (sm.rec[turn ^ 1].b >= 0) begin(sm.rec[turn ^ 1]);
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        float t = l[nt][i];
#pragma unroll
        for (int of = 4; of < 32; of <<= 1) t = __fadd_rn(t, __shfl_xor_sync(0xffffffffu, t, of));
        const int r = wr * S::kRowsPerWarp + 8 * nt + 2 * t4 + i;
        if (g == 0) {
          sm.out.m[wt * kH + half][r] = m[nt][i];
          sm.out.l[wt * kH + half][r] = t;
        }
#pragma unroll
        for (int dt = 0; dt < kI; ++dt) {
          sm.out.o[wt * kH + half][r][16 * dt + g] = o[nt][dt][i];
          sm.out.o[wt * kH + half][r][16 * dt + 8 + g] = o[nt][dt][2 + i];
        }
      }
    __syncthreads();
    if ((int)threadIdx.x < rows) {
      const int r = threadIdx.x;
      float mx = sm.out.m[0][r], ls = 0.0f;
#pragma unroll
      for (int k = 1; k < S::kParts; ++k) mx = fmaxf(mx, sm.out.m[k][r]);
      const float base = mx == -INFINITY ? 0.0f : mx;
#pragma unroll
      for (int k = 0; k < S::kParts; ++k) {
        const float f = ex2(__fsub_rn(sm.out.m[k][r], base));
        sm.out.f[k][r] = f;
        ls = __fmaf_rn(sm.out.l[k][r], f, ls);
      }
      sm.out.mx[r] = mx;
      sm.out.ls[r] = ls;
      sm.out.inv[r] = inv_of(ls);
    }
    __syncthreads();
    float* slot = partial_slot(a, blockIdx.x, sg.c0);
    const RowMap map(c, row0);
    const bool whole = sg.whole;
#pragma unroll 2
    for (int i = threadIdx.x; i < rows * (D / 4); i += S::kThreads) {
      const int r = i / (D / 4), d = i % (D / 4) * 4;
      float4 os = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
      for (int k = 0; k < S::kParts; ++k) os = fma4(*reinterpret_cast<const float4*>(&sm.out.o[k][r][d]), sm.out.f[k][r], os);
      if (whole) {
        write4<T>(a, map, sg.first, r, h, d, os, sm.out.mx[r], sm.out.ls[r], sm.out.inv[r]);
      } else {
        *reinterpret_cast<float4*>(slot + r * D + d) = os;
        if (d == 0) {
          slot[S::kRows * D + r] = sm.out.mx[r];
          slot[S::kRows * D + S::kRows + r] = sm.out.ls[r];
        }
      }
    }
    if (a.shared) {
      if (!sg.whole && sg.c0 == (int)blockIdx.x && threadIdx.x == 0)
        a.shared[blockIdx.x] = SharedTile{row0, rows, sg.first, h, sg.c1, {0, 0, 0}};
    } else if (!sg.whole) {
      __threadfence();
      __syncthreads();
      if (threadIdx.x == 0) {
        sm.last = atomicAdd(a.arrived + sg.c0, 1) == sg.c1 - sg.c0;
        if (sm.last) a.arrived[sg.c0] = 0;  // as every call leaves it
      }
      __syncthreads();
      if (sm.last) {
        __threadfence();
        for (int i = threadIdx.x; i < rows * (D / 4); i += S::kThreads) {
          const int r = i / (D / 4), d = i % (D / 4) * 4;
          // four parts at a time, their loads in flight together, each batch's
          // maximum before its sums
          float mx = -INFINITY, ls = 0.0f;
          float4 os = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
          for (int k0 = sg.c0; k0 <= sg.c1; k0 += 4) {
            float pm[4], pl[4];
            float4 po[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const float* sp = partial_slot(a, min(k0 + k, sg.c1), sg.c0);
              pm[k] = __ldcg(sp + S::kRows * D + r);
              pl[k] = __ldcg(sp + S::kRows * D + S::kRows + r);
              po[k] = __ldcg(reinterpret_cast<const float4*>(sp + r * D + d));
            }
            float mn = mx;
#pragma unroll
            for (int k = 0; k < 4; ++k) mn = fmaxf(mn, pm[k]);
            const float base = mn == -INFINITY ? 0.0f : mn, al = ex2(__fsub_rn(mx, base));
            mx = mn;
            ls = __fmul_rn(ls, al);
            os = make_float4(__fmul_rn(os.x, al), __fmul_rn(os.y, al), __fmul_rn(os.z, al), __fmul_rn(os.w, al));
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              if (k0 + k <= sg.c1) {
                const float f = ex2(__fsub_rn(pm[k], base));
                ls = __fmaf_rn(pl[k], f, ls);
                os = fma4(po[k], f, os);
              }
            }
          }
          write4<T>(a, map, sg.first, r, h, d, os, mx, ls, inv_of(ls));
        }
      }
    }
    // the next segment's values land where this one's results were
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncthreads();
  }
  if (SMALL) copies_wait();
  if (sm.dead && feeds && lane == 0) {  // copies in flight land before the block ends
    for (uint32_t i = ik > Mem::NK ? ik - Mem::NK : 0; i < ik; ++i)
      (void)mbar_wait(&sm.k_full[wt][i % Mem::NK], (i / Mem::NK) & 1, a.wait_ns);
    for (uint32_t i = iv > Mem::NV ? iv - Mem::NV : 0; i < iv; ++i)
      (void)mbar_wait(&sm.v_full[wt][i % Mem::NV], (i / Mem::NV) & 1, a.wait_ns);
  }
}

// Joins the parts of the shared tile that begins in block blockIdx.x's share. A
// block takes `RB` rows; 8 / RB warps share a row's parts, four in flight each,
// and are added in order.
template <typename T, int D, int ROWS, int RB>
__global__ void __launch_bounds__(256) paged_join_rows_kernel(const __grid_constant__ AttnArgs a) {
  constexpr int kG = 8 / RB, kV = D / 4;  // warps of a row, lanes of a part of it
  constexpr int kP = 32 / kV;             // parts a warp takes at a time
  __shared__ float4 so[8][32];
  __shared__ float sl[8][32];
  wait_for_previous();
  const SharedTile tile = a.shared[blockIdx.x];
  if ((int)blockIdx.y * RB >= tile.rows) return;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c0 = blockIdx.x;
  const int r = min((int)blockIdx.y * RB + warp / kG, tile.rows - 1), part = warp % kG;
  const int d = lane % kV * 4, sub = lane / kV;
  float m = -INFINITY, l = 0.0f;
  for (int k = c0 + lane; k <= tile.c1; k += 32) m = fmaxf(m, partial_slot(a, k, c0)[ROWS * D + r]);
#pragma unroll
  for (int i = 16; i > 0; i >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, i));
  const float base = m == -INFINITY ? 0.0f : m;
  float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 4
  for (int k = c0 + part * kP + sub; k <= tile.c1; k += kG * kP) {
    const float* sp = partial_slot(a, k, c0);
    const float f = ex2(__fsub_rn(sp[ROWS * D + r], base));
    l = __fmaf_rn(sp[ROWS * D + ROWS + r], f, l);
    o = fma4(*reinterpret_cast<const float4*>(sp + r * D + d), f, o);
  }
  so[warp][lane] = o;
  sl[warp][lane] = l;
  __syncthreads();
  if (part != 0 || sub != 0 || (int)blockIdx.y * RB + warp / kG >= tile.rows) return;
  l = 0.0f;
  o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
  for (int k = 0; k < kG * kP; ++k) {
    l = __fadd_rn(l, sl[warp + k / kP][lane + k % kP * kV]);
    o = fma4(so[warp + k / kP][lane + k % kP * kV], 1.0f, o);
  }
  write4<T>(a, RowMap(a.c, tile.row0), tile.first, r, tile.h, d, o, m, l, inv_of(l));
}

template <typename T, int D, int NT, int WR>
cudaError_t launch(const AttnArgs& a, int64_t max_blocks, cudaStream_t st) {
  const int64_t tiles = tiles_upper(a.c, Shape<NT, WR>::kRows);
  using Mem = RowsSmem<D, NT, WR>;
  static_assert((sizeof(Mem) + 1024) * Shape<NT, WR>::blocks(D) <= 228 * 1024, "shared memory of an SM");
  const auto kernel = small_pages(a.c) ? paged_rows_kernel<T, D, NT, WR, true> : paged_rows_kernel<T, D, NT, WR, false>;
  const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(Mem));
  if (e != cudaSuccess) return e;
  AttnArgs b = a;
  b.min_units = 4 * Shape<NT, WR>::kTokWarps;
  b.vec = rows_aligned(a.q, sizeof(T));
  b.vec_out = rows_aligned(a.out, sizeof(T));
  int64_t grid = 152 * Shape<NT, WR>::blocks(D);
  static_assert(152 * Shape<NT, WR>::blocks(D) <= max_attn_blocks(D), "partial results in the workspace");
  const int64_t most = tiles * a.c.kv_heads * max_blocks;
  if (grid > most) grid = most;
  // A tile of few parts is joined by its last block to arrive; where there can be
  // more, its serial reading took 40 us of a 131k-token decode step, and a second
  // launch joins all tiles on the whole GPU.
  const bool join = max_blocks / b.min_units > (Shape<NT, WR>::kRows > 16 ? 1 : kMaxParts);
  if (!join) b.shared = nullptr;
  const cudaError_t k = launch_next(kernel, dim3((unsigned)grid), Shape<NT, WR>::kThreads, sizeof(Mem), b, st);
  if (k != cudaSuccess) return k;
  note_launches(1);
  if (join) {
    constexpr int kRows = Shape<NT, WR>::kRows, kRB = kRows <= 16 ? 1 : 8;
    const cudaError_t j = launch_next(paged_join_rows_kernel<T, D, kRows, kRB>, dim3((unsigned)grid, kRows / kRB), 256, 0, b, st);
    if (j != cudaSuccess) return j;
    note_launches(1);
  }
  return cudaGetLastError();
}

template <typename T, int D>
cudaError_t pick(const AttnArgs& a, int max_new, int64_t max_blocks, cudaStream_t st) {
  const int64_t rows = (int64_t)max_new * a.c.group;
  if (rows <= 8) return launch<T, D, 1, 1>(a, max_blocks, st);
  if (rows <= 16) return launch<T, D, 2, 1>(a, max_blocks, st);
  return launch<T, D, 2, 4>(a, max_blocks, st);
}

}  // namespace

cudaError_t launch_paged_rows(const AttnArgs& a, int head_dim, int dtype, int max_new, int max_kv, cudaStream_t st) {
  const int64_t mb = max_kv > kUnit ? ((int64_t)max_kv + kUnit - 1) / kUnit : 1;
  if (dtype == AWSRC_DTYPE_BF16)
    return head_dim == 128 ? pick<__nv_bfloat16, 128>(a, max_new, mb, st) : pick<__nv_bfloat16, 64>(a, max_new, mb, st);
  return head_dim == 128 ? pick<float, 128>(a, max_new, mb, st) : pick<float, 64>(a, max_new, mb, st);
}

}  // namespace awsrc
