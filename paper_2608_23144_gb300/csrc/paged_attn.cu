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
// the second term costs one more MMA on the same codes.
//
// Bound by the cache's bytes when rows are few. A warp takes 64 tokens at a
// time: its lanes read 16-byte runs straight into MMA fragments (the cache's
// byte order is chosen for that), the order of tokens and dims inside the
// fragments being free as long as both operands agree.
//
// Work: the (sequence, row tile, kv head, 64-token block) units of the batch in
// this order are dealt out in equal contiguous shares to the thread blocks,
// whatever the lengths. A tile that several blocks share is joined in block order
// from partial results in the workspace, by its last block to arrive or by a
// second launch; nothing waits.
#include "internal.h"
#include "kv_paged.cuh"

namespace awsrc {

namespace {

constexpr int kThreads = 128;
constexpr int kWarps = kThreads / 32;
constexpr int kUnit = 64;         // tokens per unit
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kPBits = 15.0f;   // p is at most 2^15
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

__device__ __forceinline__ uint4 ldg16(const uint8_t* p) { return __ldg(reinterpret_cast<const uint4*>(p)); }

template <typename T>
__device__ __forceinline__ float elem(const T* p);
template <>
__device__ __forceinline__ float elem(const float* p) { return __ldg(p); }
template <>
__device__ __forceinline__ float elem(const __nv_bfloat16* p) { return __bfloat162float(*p); }

template <int NT, int WR>
struct Shape {
  static constexpr int kRowsPerWarp = 8 * NT;
  static constexpr int kRows = kRowsPerWarp * WR;  // query rows of a tile
  static constexpr int kTokWarps = kWarps / WR;    // warps that share the tokens of a row group
};

template <int D>
struct RowStride { static constexpr int value = D + 4; };  // floats of a row in shared memory

// Element d of row r of a finished tile, and its lse.
template <typename T, int D>
__device__ __forceinline__ void write_final(const AttnArgs& a, const KvSeq& s, int row, int h, int d, float o, float m,
                                            float l) {
  const int tok = s.first + row / a.c.group, head = h * a.c.group + row % a.c.group;
  const float v = l == 0.0f ? 0.0f : __fdiv_rn(o, l);
  T* p = static_cast<T*>(a.out.p) + (int64_t)tok * a.out.ts + (int64_t)head * a.out.hs + d;
  if constexpr (sizeof(T) == 2)
    *p = __float2bfloat16_rn(v);
  else
    *p = v;
  if (d == 0 && a.lse)
    a.lse[(int64_t)tok * a.c.n_heads + head] = l == 0.0f ? -INFINITY : (m - kPBits + log2f(l)) * kLn2;
}

struct Place {
  int jk, pk, ek, ev;
  bool kbad, pad_;
};

template <typename T, int D, int NT, int WR>
__global__ void __launch_bounds__(kThreads, 2) paged_rows_kernel(const __grid_constant__ AttnArgs a) {
  using S = Shape<NT, WR>;
  constexpr bool kSplit = sizeof(T) == 4;
  constexpr int kTerms = kSplit ? 2 : 1;
  constexpr int kC = D / 64;           // 16-byte runs of a token's dims per lane
  constexpr int kStride = RowStride<D>::value;
  constexpr bool kAhead = NT == 1;     // registers for a block's keys and values ahead of their use
  __shared__ float so[S::kTokWarps][S::kRows][kStride];
  __shared__ float sm[S::kTokWarps][S::kRows], sl[S::kTokWarps][S::kRows];
  __shared__ int last_flag;
  const KvArgs& c = a.c;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int g = lane >> 2, t4 = lane & 3;
  const int wr = warp % WR, wt = warp / WR;

  UnitWalk<S::kRows, kUnit, kWarps, 0> w;
  SharedTile mine{};
  if (!w.start(a)) {
    if (a.shared && threadIdx.x == 0) a.shared[blockIdx.x] = mine;
    return;
  }
  while (w.more()) {
    const Segment sg = w.segment(a);
    const KvSeq s = w.s;
    const int h = sg.h, rows = sg.rows, row0 = w.t * S::kRows;
    const int32_t* table = c.table + (int64_t)w.b * c.table_stride;

    // ---- query fragments: row r0 + 8 nt + g, dims 16 t4 .. + 15 (+ 64)
    uint32_t qf[NT][kTerms][kC * 8];
    float rm[NT][2];     // score multiplier of rows 2 t4, 2 t4 + 1
    int lim[NT][2];      // last token these rows see
    int lim_min = INT32_MAX;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int r = wr * S::kRowsPerWarp + 8 * nt + g;
      const int row = row0 + r;
      const bool have = r < rows;
      const int tok = row / c.group;
      float x[kC * 16];
      if (have) {
        const T* p = static_cast<const T*>(a.q.p) + (int64_t)(s.first + tok) * a.q.ts +
                     (int64_t)(h * c.group + row % c.group) * a.q.hs + 16 * t4;
#pragma unroll
        for (int i = 0; i < kC; ++i)
#pragma unroll
          for (int j = 0; j < 16; ++j) x[16 * i + j] = elem<T>(p + 64 * i + j);
      } else {
#pragma unroll
        for (int i = 0; i < kC * 16; ++i) x[i] = 0.0f;
      }
      float amax = 0.0f;
#pragma unroll
      for (int i = 0; i < kC * 16; ++i) amax = fmaxf(amax, fabsf(x[i]));
      amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 1));
      amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 2));
      // the row times 2^up has its largest element in [2^14, 2^15)
      const int ex = (int)(__float_as_uint(amax) >> 23) - 127;
      const int up = min(max(14 - ex, -120), 100);
      const float f = pow2f(up), mul = a.score_mul * pow2f(-up);
#pragma unroll
      for (int i = 0; i < kC * 8; ++i) {
        const float y0 = __fmul_rn(x[2 * i], f), y1 = __fmul_rn(x[2 * i + 1], f);
        qf[nt][0][i] = half2_bits(y0, y1);
        if constexpr (kSplit) {
          const float2 hi = half2_floats(qf[nt][0][i]);
          qf[nt][1][i] = half2_bits(__fsub_rn(y0, hi.x), __fsub_rn(y1, hi.y));
        }
      }
      const int see = a.causal ? s.kv - s.n + tok : s.kv - 1;
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

    float o[NT][D / 16][4], m[NT][2], l[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
      for (int i = 0; i < 2; ++i) m[nt][i] = -INFINITY, l[nt][i] = 0.0f;
#pragma unroll
      for (int dt = 0; dt < D / 16; ++dt)
#pragma unroll
        for (int i = 0; i < 4; ++i) o[nt][dt][i] = 0.0f;
    }

    // Page and block exponents of this lane's key tokens (16-token group g / 2 of
    // a block; its value tokens' page, group t4, comes by shuffle).
    auto find = [&](int blk) {
      Place p{0, 0, 0, 0, false, false};
      p.jk = blk * kUnit + 16 * (g >> 1);
      if (blk < sg.blk1 && p.jk < s.kv) p.pk = __ldg(table + (p.jk >> c.log_page));
      p.kbad = p.pk < 0 || p.pk >= c.n_pages;
      if (p.kbad) {
        atomicOr(c.status, kFaultBatch);
        p.pk = 0;
      }
      p.ek = __ldg(c.k_exp + (int64_t)p.pk * c.kv_heads + h);
      p.ev = __ldg(c.v_exp + (int64_t)p.pk * c.kv_heads + h);
      return p;
    };
    // Key bytes of MMA row tile i (16 tokens; rows 0-7: tokens 16 (g / 2) + 4 i +
    // g % 2, rows 8-15: two further), 16 dims at 16 t4 (+ 64).
    uint4 kreg[4][kC][2];
    auto load_keys = [&](const Place& p, int i) {
      const uint8_t* kb = c.k + block_off<D>(c, p.pk, h);
      const int row = (p.jk & (c.page - 1)) + 4 * i + (g & 1);
#pragma unroll
      for (int cc = 0; cc < kC; ++cc) {
        const uint8_t* kp = kb + ((((t4 + 4 * cc) << c.log_page) + row) << 4);
        kreg[i][cc][0] = ldg16(kp);
        kreg[i][cc][1] = ldg16(kp + 32);
      }
    };
    Place next = find(sg.blk0 + wt);
    if (kAhead) {
#pragma unroll
      for (int i = 0; i < 4; ++i) load_keys(next, i);
    }
    for (int blk = sg.blk0 + wt; blk < sg.blk1; blk += S::kTokWarps) {
      const Place cur = next;
      const bool bad = cur.kbad;
      const int jk = cur.jk, jv = blk * kUnit + 16 * t4, ek = cur.ek, ev = cur.ev;
      next = find(blk + S::kTokWarps);
      const bool vbad = __shfl_sync(0xffffffffu, bad, 8 * t4);
      const int pv = __shfl_sync(0xffffffffu, cur.pk, 8 * t4);
      const uint8_t* vb = c.v + block_off<D>(c, pv, h) + (((int64_t)((jv & (c.page - 1)) >> 4) * D) << 4);
      // value bytes of 8 + 8 dims per MMA row tile, 16 tokens of group t4
      uint4 vreg[D / 16][2];
      auto load_values = [&](int dt) {
        const uint8_t* vp = vb + ((16 * dt + g) << 4);
        vreg[dt][0] = ldg16(vp);
        vreg[dt][1] = ldg16(vp + 128);
      };
      if (kAhead) {
#pragma unroll
        for (int dt = 0; dt < D / 16; ++dt) load_values(dt);
      }

      // ---- scores
      float x[NT][4][4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int j = 0; j < 4; ++j) x[nt][i][j] = 0.0f;
        if (!kAhead) load_keys(cur, i);
#pragma unroll
        for (int cc = 0; cc < kC; ++cc) {
          uint32_t f0[8], f1[8];
          widen(kreg[i][cc][0], f0);
          widen(kreg[i][cc][1], f1);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const uint32_t fr[4] = {f0[2 * j], f1[2 * j], f0[2 * j + 1], f1[2 * j + 1]};
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
              for (int q = kTerms - 1; q >= 0; --q)
                mma(x[nt][i], fr, qf[nt][q][8 * cc + 2 * j], qf[nt][q][8 * cc + 2 * j + 1]);
          }
        }
      }
      if (kAhead && blk + S::kTokWarps < sg.blk1) {  // the next block's keys load under the rest of this one
#pragma unroll
        for (int i = 0; i < 4; ++i) load_keys(next, i);
      }

      // ---- softmax weights; this lane's tokens lie in one block
      const float nan = __int_as_float(0x7FC00000);
      const float sk = ek == kExpNan ? nan : pow2f(ek), evf = ev == kExpNan ? nan : (float)ev;
      const float un = ev == kExpNan ? nan : pow2f(-ev);
      const bool masked = blk * kUnit + kUnit - 1 > lim_min || __any_sync(0xffffffffu, bad);
      uint32_t pf[NT][kTerms][8];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        float mx[2] = {-INFINITY, -INFINITY};
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const float k = __fmul_rn(rm[nt][i], sk);
#pragma unroll
          for (int s = 0; s < 4; ++s)
#pragma unroll
            for (int hf = 0; hf < 2; ++hf) {
              float y = __fmaf_rn(x[nt][s][2 * hf + i], k, evf);
              if (masked && (bad || jk + 4 * s + (g & 1) + 2 * hf > lim[nt][i])) y = -INFINITY;
              x[nt][s][2 * hf + i] = y;
              mx[i] = fmaxf(mx[i], y);
            }
#pragma unroll
          for (int of = 4; of < 32; of <<= 1) mx[i] = fmaxf(mx[i], __shfl_xor_sync(0xffffffffu, mx[i], of));
          const float mn = fmaxf(m[nt][i], mx[i]);
          const float base = mn == -INFINITY ? 0.0f : mn;
          const float al = ex2(__fsub_rn(m[nt][i], base));
          m[nt][i] = mn;
          float sum = 0.0f;
#pragma unroll
          for (int s = 0; s < 4; ++s)
#pragma unroll
            for (int hf = 0; hf < 2; ++hf) {
              const float p = ex2(__fsub_rn(x[nt][s][2 * hf + i], __fsub_rn(base, kPBits)));
              x[nt][s][2 * hf + i] = p;
              sum = __fadd_rn(sum, p);
            }
          l[nt][i] = __fmaf_rn(l[nt][i], al, sum == 0.0f ? 0.0f : __fmul_rn(sum, un));
#pragma unroll
          for (int dt = 0; dt < D / 16; ++dt) {
            o[nt][dt][i] = __fmul_rn(o[nt][dt][i], al);
            o[nt][dt][2 + i] = __fmul_rn(o[nt][dt][2 + i], al);
          }
        }
#pragma unroll
        for (int s = 0; s < 4; ++s)
#pragma unroll
          for (int hf = 0; hf < 2; ++hf) {
            const float p0 = x[nt][s][2 * hf], p1 = x[nt][s][2 * hf + 1];
            const uint32_t hi = half2_bits(p0, p1);
            pf[nt][0][2 * s + hf] = transpose8(hi);
            if constexpr (kSplit) {
              const float2 b = half2_floats(hi);
              pf[nt][1][2 * s + hf] = transpose8(half2_bits(__fsub_rn(p0, b.x), __fsub_rn(p1, b.y)));
            }
          }
      }

      // ---- O^T += V^T P^T: MMA row tiles of 16 dims, 4 steps of 16 tokens.
      // Rows that hold no token yet may hold any bytes, e4m3's NaN among them.
      const bool tail = masked && (blk * kUnit + kUnit > s.kv || __any_sync(0xffffffffu, vbad));
      uint4 keep = make_uint4(~0u, ~0u, ~0u, ~0u);
      if (tail) {
        const int have = vbad ? 0 : s.kv - jv;
        keep.x = first_bytes(have);
        keep.y = first_bytes(have - 4);
        keep.z = first_bytes(have - 8);
        keep.w = first_bytes(have - 12);
      }
#pragma unroll
      for (int dt = 0; dt < D / 16; ++dt) {
        if (!kAhead) load_values(dt);
        uint4 v0 = vreg[dt][0], v1 = vreg[dt][1];
        if (tail) {
          v0 = make_uint4(v0.x & keep.x, v0.y & keep.y, v0.z & keep.z, v0.w & keep.w);
          v1 = make_uint4(v1.x & keep.x, v1.y & keep.y, v1.z & keep.z, v1.w & keep.w);
        }
        uint32_t f0[8], f1[8];
        widen(v0, f0);
        widen(v1, f1);
#pragma unroll
        for (int s = 0; s < 4; ++s) {
          const uint32_t fr[4] = {f0[2 * s], f1[2 * s], f0[2 * s + 1], f1[2 * s + 1]};
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int q = kTerms - 1; q >= 0; --q) mma(o[nt][dt], fr, pf[nt][q][2 * s], pf[nt][q][2 * s + 1]);
        }
      }
    }

    // ---- the warps' results to shared memory
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        float t = l[nt][i];
#pragma unroll
        for (int of = 4; of < 32; of <<= 1) t = __fadd_rn(t, __shfl_xor_sync(0xffffffffu, t, of));
        const int r = wr * S::kRowsPerWarp + 8 * nt + 2 * t4 + i;
        if (g == 0) {
          sm[wt][r] = m[nt][i];
          sl[wt][r] = t;
        }
#pragma unroll
        for (int dt = 0; dt < D / 16; ++dt) {
          so[wt][r][16 * dt + g] = o[nt][dt][i];
          so[wt][r][16 * dt + 8 + g] = o[nt][dt][2 + i];
        }
      }
    __syncthreads();

    float* slot = partial_slot(a, blockIdx.x, sg.c0);
    for (int i = threadIdx.x; i < rows * D; i += kThreads) {
      const int r = i / D, d = i % D;
      float mx = sm[0][r];
#pragma unroll
      for (int k = 1; k < S::kTokWarps; ++k) mx = fmaxf(mx, sm[k][r]);
      const float base = mx == -INFINITY ? 0.0f : mx;
      float os = 0.0f, ls = 0.0f;
#pragma unroll
      for (int k = 0; k < S::kTokWarps; ++k) {
        const float f = ex2(__fsub_rn(sm[k][r], base));
        os = __fmaf_rn(so[k][r][d], f, os);
        ls = __fmaf_rn(sl[k][r], f, ls);
      }
      if (sg.whole) {
        write_final<T, D>(a, s, row0 + r, h, d, os, mx, ls);
      } else {
        slot[r * D + d] = os;
        if (d == 0) {
          slot[S::kRows * D + r] = mx;
          slot[S::kRows * D + S::kRows + r] = ls;
        }
      }
    }
    if (a.shared) {
      if (!sg.whole && sg.c0 == (int)blockIdx.x) mine = SharedTile{row0, rows, s.first, h, sg.c1, {0, 0, 0}};
    } else if (!sg.whole) {
      __threadfence();
      __syncthreads();
      if (threadIdx.x == 0) {
        last_flag = atomicAdd(a.arrived + sg.c0, 1) == sg.c1 - sg.c0;
        if (last_flag) a.arrived[sg.c0] = 0;  // as every call leaves it
      }
      __syncthreads();
      if (last_flag) {
        __threadfence();
        for (int i = threadIdx.x; i < rows * D; i += kThreads) {
          const int r = i / D, d = i % D;
          float mx = -INFINITY;
#pragma unroll 4
          for (int k = sg.c0; k <= sg.c1; ++k) mx = fmaxf(mx, __ldcg(partial_slot(a, k, sg.c0) + S::kRows * D + r));
          const float base = mx == -INFINITY ? 0.0f : mx;
          float os = 0.0f, ls = 0.0f;
#pragma unroll 4
          for (int k = sg.c0; k <= sg.c1; ++k) {
            const float* sp = partial_slot(a, k, sg.c0);
            const float f = ex2(__fsub_rn(__ldcg(sp + S::kRows * D + r), base));
            os = __fmaf_rn(__ldcg(sp + r * D + d), f, os);
            ls = __fmaf_rn(__ldcg(sp + S::kRows * D + S::kRows + r), f, ls);
          }
          write_final<T, D>(a, s, row0 + r, h, d, os, mx, ls);
        }
      }
    }
    __syncthreads();  // shared memory is free for the next segment

    w.advance(a, sg);
  }
  if (a.shared && threadIdx.x == 0) a.shared[blockIdx.x] = mine;
}

// Joins the parts of the shared tile that begins in block blockIdx.x's share. A
// block takes `RB` rows; 8 / RB warps share a row's parts, four in flight each,
// and are added in order.
template <typename T, int D, int ROWS, int RB>
__global__ void __launch_bounds__(256) paged_join_rows_kernel(const __grid_constant__ AttnArgs a) {
  constexpr int kG = 8 / RB, kV = D / 32;  // warps of a row, dims of a lane
  __shared__ float so[8][D], sml[8][2];
  const SharedTile tile = a.shared[blockIdx.x];
  if ((int)blockIdx.y * RB >= tile.rows) return;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c0 = blockIdx.x;
  const int r = min((int)blockIdx.y * RB + warp / kG, tile.rows - 1), part = warp % kG;
  float m = -INFINITY, l = 0.0f, o[kV];
  for (int k = c0 + lane; k <= tile.c1; k += 32) m = fmaxf(m, partial_slot(a, k, c0)[ROWS * D + r]);
#pragma unroll
  for (int i = 16; i > 0; i >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, i));
  const float base = m == -INFINITY ? 0.0f : m;
#pragma unroll
  for (int j = 0; j < kV; ++j) o[j] = 0.0f;
#pragma unroll 4
  for (int k = c0 + part; k <= tile.c1; k += kG) {
    const float* sp = partial_slot(a, k, c0);
    const float f = ex2(__fsub_rn(sp[ROWS * D + r], base));
    l = __fmaf_rn(sp[ROWS * D + ROWS + r], f, l);
#pragma unroll
    for (int j = 0; j < kV; ++j) o[j] = __fmaf_rn(sp[r * D + 32 * j + lane], f, o[j]);
  }
#pragma unroll
  for (int j = 0; j < kV; ++j) so[warp][32 * j + lane] = o[j];
  if (lane == 0) sml[warp][0] = l;
  __syncthreads();
  if (part != 0 || (int)blockIdx.y * RB + warp / kG >= tile.rows) return;
  // l of the row first, then its dims
  l = 0.0f;
#pragma unroll
  for (int k = 0; k < kG; ++k) l = __fadd_rn(l, sml[warp + k][0]);
  KvSeq s{tile.first, 0, 0};
#pragma unroll
  for (int j = 0; j < kV; ++j) {
    float v = 0.0f;
#pragma unroll
    for (int k = 0; k < kG; ++k) v = __fadd_rn(v, so[warp + k][32 * j + lane]);
    write_final<T, D>(a, s, tile.row0 + r, tile.h, 32 * j + lane, v, m, l);
  }
}

template <typename T, int D, int NT, int WR>
cudaError_t launch(const AttnArgs& a, int64_t max_blocks, cudaStream_t st) {
  const int64_t tiles = tiles_upper(a.c, Shape<NT, WR>::kRows);
  AttnArgs b = a;
  b.min_units = Shape<NT, WR>::kTokWarps;
  int64_t grid = kMaxAttnBlocks;
  const int64_t most = tiles * a.c.kv_heads * max_blocks;
  if (grid > most) grid = most;
  // A tile of few parts is joined by its last block to arrive; where there can be
  // more, its serial reading took 40 us of a 131k-token decode step, and a second
  // launch joins all tiles on the whole GPU.
  const bool join = max_blocks / b.min_units > kMaxParts;
  if (!join) b.shared = nullptr;
  paged_rows_kernel<T, D, NT, WR><<<(unsigned)grid, kThreads, 0, st>>>(b);
  note_launches(1);
  if (join) {
    constexpr int kRows = Shape<NT, WR>::kRows, kRB = kRows <= 16 ? 1 : 8;
    paged_join_rows_kernel<T, D, kRows, kRB><<<dim3((unsigned)grid, kRows / kRB), 256, 0, st>>>(b);
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
