// paged_tiles.cu — BF16 attention of many query rows per kv head over the paged
// 8-bit cache (prompts, chunks, drafts, also beside single tokens) on the
// fifth-generation tensor cores.
//
// Mathematics as in paged_attn.cu: base-2 scores x = (q . k) 2^ek sm_scale
// log2(e) + ev, weights p = 2^(x - m + 6) with m a maximum seen so far, O = sum
// p c over the value codes, l = sum p 2^-ev.
//
// Precision at the cost of one 16-bit product each:
//   q . k   kind::f8f6f4 on the key codes as they lie in the cache; q, scaled by
//           a power of two per row, is split into two e4m3 terms, which hold the
//           8 significant bits of a bf16 (two 8-bit products cost what one
//           16-bit product costs; no key is ever converted);
//   p . V   kind::f16 with p in binary16 (from tensor memory) and the value
//           codes widened to binary16, exactly, by four warps. Splitting p into
//           8-bit terms instead would cost the softmax warps two more
//           conversions per weight, five times the widening's instructions.
// Floor: 4 D flop per (row, token) at the bf16 rate.
//
// One thread block per SM and 256 rows (query tokens x the heads of a kv head)
// in two tiles of 128, so that one tile's softmax runs under the other's
// products. Warps 0-3 and 4-7: softmax, one row per thread; 8-11: widening; 12:
// MMA issue; 13: bulk copies. Tensor memory: S 2 x 128 columns, over whose
// first 64 P is written; O 2 x D columns. Per tile and block of 128 tokens:
//   MMA:     P ready -> O += P V; S = Q K of the next block -> commit
//   softmax: S ready -> m, P, l; O rescaled by its own threads, only when a row
//            grew by more than 2^8 (the commit that made S ready also covers
//            the products that wrote O).
// The byte order of keys and values in the cache is the operand order the
// tensor cores read, so copies need no rearrangement.
//
// Work is shared out as in paged_attn.cu (UnitWalk); tiles that thread blocks
// share are joined by the last to arrive.
//
// Every wait is bounded (wait_ns): one that runs out sets bit 2 of the fault
// word, stops the block's roles, waits (bounded) for its copies and products in
// flight and frees the tensor memory.
#include "internal.h"
#include "kv_paged.cuh"
#include "tc05.cuh"

namespace awsrc {

namespace {

using namespace tc05;

constexpr int BM = 128, BN = 128;
constexpr int kRows = 2 * BM;
constexpr int kThreads = 448;
constexpr int kMmaWarp = 12, kLoadWarp = 13;
constexpr int NK = 3, NV = 2, NW = 2;  // stages: keys, value codes, widened values
constexpr uint32_t kTmemCols = 512;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kPBits = 6.0f;         // p is at most 2^6 when m is the maximum,
constexpr float kGrow = 8.0f;          // and at most 2^(6 + 8) < 65504 when m lags
using Walk = UnitWalk<kRows, BN, 4>;

template <int N>
struct Idesc { static constexpr uint32_t value = idesc_f16(BM, N); };  // formats 0: e4m3, binary16

template <int D>
struct Smem {
  uint8_t q[2][2][D / 16][BM][16];  // tile, term, 16 dims
  uint8_t k[NK][D / 16][BN][16];
  uint8_t v[NV][BN / 16][D][16];
  uint8_t w[NW][BN / 8][D][16];     // binary16, 8 tokens
  unsigned long long k_full[NK], k_empty[NK], v_full[NV], v_empty[NV], w_full[NW], w_empty[NW];
  unsigned long long q_full[2], s_full[2], p_full[2], o_full[2], group[2], drain;
  uint32_t tmem;
  int dead, last[2];
};

struct Ctx {
  uint64_t wait_ns;
  uint32_t* status;
  volatile int* dead;
};

// Bounded wait of a whole warp; false, for all lanes, once any wait of the
// block has given up.
__device__ __noinline__ bool wait_slow(const Ctx& x, unsigned long long* mb, uint32_t parity) {
  const uint64_t t0 = globaltimer();
  bool ok;
  for (;;) {
    ok = mbar_try_wait(mb, parity);
    if (ok || *x.dead) break;
    if (globaltimer() - t0 > x.wait_ns) {
      *x.dead = 1;
      atomicOr(x.status, kFaultTimeout);
      break;
    }
  }
  return ok;
}
__device__ __forceinline__ bool wait_warp(const Ctx& x, unsigned long long* mb, uint32_t parity) {
  bool ok = mbar_try_wait(mb, parity);
  if (!__all_sync(0xffffffffu, ok)) {
    ok = wait_slow(x, mb, parity);
    if (!__all_sync(0xffffffffu, ok)) return false;
  }
  return true;
}
__device__ __forceinline__ bool wait_lane(const Ctx& x, unsigned long long* mb, uint32_t parity) {
  return mbar_try_wait(mb, parity) || wait_slow(x, mb, parity);
}

// K-major operand without swizzle: 8 rows x 16 bytes core matrices, 128 B apart
// along the rows, kbytes along the reduced axis.
__device__ __forceinline__ uint64_t desc(uint32_t addr, uint32_t kbytes) {
  return (uint64_t)((addr & 0x3FFFFu) >> 4) | ((uint64_t)(kbytes >> 4) << 16) | ((uint64_t)(128u >> 4) << 32) |
         (1ull << 46);
}

// D(tmem) (+)= A(smem, e4m3) B(smem, e4m3), 32 deep.
__device__ __forceinline__ void umma_f8(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"(accumulate)
      : "memory");
}
// D(tmem) (+)= A(tmem, binary16) B(smem, binary16), 16 deep.
__device__ __forceinline__ void umma_f16_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
      "r"(a), "l"(b), "r"(idesc), "r"(accumulate)
      : "memory");
}

// 16 consecutive columns of the warp's 32 lanes; ready after st_wait().
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], "
      "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15};" ::"r"(r[0]),
      "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
      "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(taddr)
      : "memory");
}
__device__ __forceinline__ void st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// What the lanes of a warp know about the eight 16-token groups of a block,
// lane i < 8 about group i: tokens in it (0 for a page that cannot be right)
// and the exponents of its page.
struct Groups {
  int page, have, ek, ev;
};
__device__ __forceinline__ Groups load_groups(const KvArgs& c, const int32_t* table, int kv, int h, int blk) {
  const int lane = threadIdx.x & 31;
  const int j = blk * BN + 16 * (lane & 7);
  Groups g{0, 0, 0, 0};
  if (lane < 8 && j < kv) {
    const int pg = __ldg(table + (j >> c.log_page));
    if (pg >= 0 && pg < c.n_pages) {
      g.page = pg;
      g.have = min(16, kv - j);
      g.ek = __ldg(c.k_exp + (int64_t)pg * c.kv_heads + h);
      g.ev = __ldg(c.v_exp + (int64_t)pg * c.kv_heads + h);
    }
  }
  return g;
}

// ------------------------------------------------------------------- copies --
template <int D>
__device__ void load_role(const AttnArgs& a, Walk w, Smem<D>& sm, const Ctx& x) {
  const KvArgs& c = a.c;
  const int lane = threadIdx.x & 31;
  const int per = BN >> c.log_page;  // pages of a block
  uint32_t n = 0;
  bool ok = true;
  while (ok && w.more()) {
    const Segment sg = w.segment(a);
    const int32_t* table = c.table + (int64_t)w.b * c.table_stride;
    for (int blk = sg.blk0; ok && blk < sg.blk1; ++blk, ++n) {
      if ((int)n == a.stall) {  // the limit's test
        ok = false;
        break;
      }
      // lane i < per: page i of the block
      int pg = -1;
      const int j = blk * BN + (lane << c.log_page);
      if (lane < per && j < w.s.kv) {
        pg = __ldg(table + (j >> c.log_page));
        if (pg < 0 || pg >= c.n_pages) {
          atomicOr(c.status, kFaultBatch);
          pg = -1;
        }
      }
      const uint32_t bytes = (uint32_t)(__popc(__ballot_sync(0xffffffffu, pg >= 0)) * D) << c.log_page;
      const int ks = n % NK, vs = n % NV;
      if (!(ok = wait_warp(x, &sm.k_empty[ks], ((n / NK) & 1) ^ 1))) break;
      if (lane == 0) mbar_expect_tx(&sm.k_full[ks], bytes);
      __syncwarp();
      for (int i0 = 0; i0 < (D / 16) * per; i0 += 32) {
        const int i = i0 + lane, p = i & (per - 1), run = i / per;
        const int pp = __shfl_sync(0xffffffffu, pg, p);
        if (pp >= 0 && run < D / 16)
          bulk_g2s(&sm.k[ks][run][p << c.log_page][0], c.k + block_off<D>(c, pp, sg.h) + ((run << c.log_page) << 4),
                   16u << c.log_page, &sm.k_full[ks]);
      }
      if (!(ok = wait_warp(x, &sm.v_empty[vs], ((n / NV) & 1) ^ 1))) {
        ++n;
        break;
      }
      if (lane == 0) mbar_expect_tx(&sm.v_full[vs], bytes);
      __syncwarp();
      if (pg >= 0)
        bulk_g2s(&sm.v[vs][(lane << c.log_page) >> 4][0][0], c.v + block_off<D>(c, pg, sg.h), (uint32_t)D << c.log_page,
                 &sm.v_full[vs]);
      __syncwarp();
    }
    if (ok) w.advance(a, sg);
  }
  if (!ok && lane == 0) {  // copies in flight land before the block ends
    for (uint32_t j = n > NK ? n - NK : 0; j < n; ++j) (void)mbar_wait(&sm.k_full[j % NK], (j / NK) & 1, x.wait_ns);
    for (uint32_t j = n > NV ? n - NV : 0; j < n; ++j) (void)mbar_wait(&sm.v_full[j % NV], (j / NV) & 1, x.wait_ns);
  }
}

// ----------------------------------------------------------------- products --
template <int D>
__device__ void mma_role(const AttnArgs& a, Walk w, Smem<D>& sm, const Ctx& x) {
  constexpr uint32_t kIdescS = Idesc<BN>::value, kIdescO = Idesc<D>::value;
  const uint32_t tmem = sm.tmem;
  uint32_t n = 0, np[2] = {0, 0}, nq[2] = {0, 0};
  auto qk = [&](int t, uint32_t blk) {
    const uint32_t kb = smem_addr(&sm.k[blk % NK][0][0][0]);
#pragma unroll
    for (int term = 0; term < 2; ++term) {
      const uint32_t qb = smem_addr(&sm.q[t][term][0][0][0]);
#pragma unroll
      for (int s = 0; s < D / 32; ++s)
        umma_f8(tmem + t * BN, desc(qb + s * 2 * BM * 16, BM * 16), desc(kb + s * 2 * BN * 16, BN * 16), kIdescS,
                term + s > 0);
    }
    umma_commit(&sm.s_full[t]);
  };
  bool ok = true;
  while (ok && w.more()) {
    const Segment sg = w.segment(a);
    const int nt = sg.rows > BM ? 2 : 1, nb = sg.blk1 - sg.blk0;
    for (int t = 0; ok && t < nt; ++t) ok = wait_lane(x, &sm.q_full[t], nq[t]++ & 1);
    if (!ok || !(ok = wait_lane(x, &sm.k_full[n % NK], (n / NK) & 1))) break;
    tc_fence_after();
    for (int t = 0; t < nt; ++t) qk(t, n);
    umma_commit(&sm.k_empty[n % NK]);
    for (int i = 0; ok && i < nb; ++i, ++n) {
      const uint32_t n1 = n + 1;
      if (i + 1 < nb && !(ok = wait_lane(x, &sm.k_full[n1 % NK], (n1 / NK) & 1))) break;
      if (!(ok = wait_lane(x, &sm.w_full[n % NW], (n / NW) & 1))) break;
      const uint32_t vb = smem_addr(&sm.w[n % NW][0][0][0]);
      for (int t = 0; t < nt; ++t) {
        if (!(ok = wait_lane(x, &sm.p_full[t], np[t]++ & 1))) break;
        tc_fence_after();
#pragma unroll
        for (int s = 0; s < BN / 16; ++s)
          umma_f16_ts(tmem + 2 * BN + t * D, tmem + t * BN + s * 8, desc(vb + s * 2 * D * 16, D * 16), kIdescO,
                      i + s > 0);
        if (i + 1 < nb)
          qk(t, n1);
        else
          umma_commit(&sm.o_full[t]);
      }
      if (!ok) break;
      umma_commit(&sm.w_empty[n % NW]);
      if (i + 1 < nb) umma_commit(&sm.k_empty[n1 % NK]);
    }
    if (ok) w.advance(a, sg);
  }
  if (!ok) {  // products in flight end before the block does
    umma_commit(&sm.drain);
    (void)mbar_wait(&sm.drain, 0, x.wait_ns);
  }
}

// ----------------------------------------------------------------- widening --
template <int D>
__device__ void widen_role(const AttnArgs& a, Walk w, Smem<D>& sm, const Ctx& x) {
  const KvArgs& c = a.c;
  const int tid = threadIdx.x & 127;
  uint32_t n = 0;
  bool ok = true;
  while (ok && w.more()) {
    const Segment sg = w.segment(a);
    const int32_t* table = c.table + (int64_t)w.b * c.table_stride;
    for (int blk = sg.blk0; blk < sg.blk1; ++blk, ++n) {
      const Groups g = load_groups(c, table, w.s.kv, sg.h, blk);
      // rows that hold no token may hold any bytes, e4m3's NaN among them: zeros
      const bool tail = __any_sync(0xffffffffu, (threadIdx.x & 31) < 8 && g.have < 16);
      if (!(ok = wait_warp(x, &sm.v_full[n % NV], (n / NV) & 1)) ||
          !(ok = wait_warp(x, &sm.w_empty[n % NW], ((n / NW) & 1) ^ 1)))
        break;
      const uint8_t* src = &sm.v[n % NV][0][0][0];
      uint8_t* dst = &sm.w[n % NW][0][0][0];
#pragma unroll
      for (int i = 0; i < BN / 16 * D / 128; ++i) {
        const int e = tid + 128 * i, run = e / D, d = e % D;
        uint4 v = *reinterpret_cast<const uint4*>(src + (size_t)e * 16);
        if (tail) {
          const int have = __shfl_sync(0xffffffffu, g.have, run);
          v.x &= first_bytes(have);
          v.y &= first_bytes(have - 4);
          v.z &= first_bytes(have - 8);
          v.w &= first_bytes(have - 12);
        }
        uint32_t f[8];
        widen(v, f);
        *reinterpret_cast<uint4*>(dst + (size_t)((2 * run) * D + d) * 16) = make_uint4(f[0], f[1], f[2], f[3]);
        *reinterpret_cast<uint4*>(dst + (size_t)((2 * run + 1) * D + d) * 16) = make_uint4(f[4], f[5], f[6], f[7]);
      }
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      mbar_arrive(&sm.w_full[n % NW]);
      mbar_arrive(&sm.v_empty[n % NV]);
    }
    if (ok) w.advance(a, sg);
  }
}

// ------------------------------------------------------------------ softmax --
__device__ __forceinline__ void load_q8(const __nv_bfloat16* p, bool vec, float* y) {
  if (vec) {
    const uint4 v = __ldg(reinterpret_cast<const uint4*>(p));
    const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      y[2 * j] = __uint_as_float(u[j] << 16);
      y[2 * j + 1] = __uint_as_float(u[j] & 0xFFFF0000u);
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) y[j] = __bfloat162float(p[j]);
  }
}

// Row r of tile t -> its query row as two e4m3 terms in shared memory; returns
// the multiplier of its scores.
template <int D>
__device__ float stage_q(const AttnArgs& a, Smem<D>& sm, int t, int r, const __nv_bfloat16* p) {
  const bool vec = reinterpret_cast<uintptr_t>(p) % 16 == 0;
  float amax = 0.0f;
  if (p != nullptr) {
#pragma unroll 4
    for (int i = 0; i < D / 8; ++i) {
      float y[8];
      load_q8(p + 8 * i, vec, y);
#pragma unroll
      for (int j = 0; j < 8; ++j) amax = fmax_nan(amax, fabsf(y[j]));
    }
  }
  // the row times 2^up has its largest element in [2^7, 2^8)
  const int ex = (int)(__float_as_uint(amax) >> 23) - 127;
  const int up = min(max(7 - ex, -120), 100);
  const float f = a.score_mul < 0.0f ? -pow2f(up) : pow2f(up);
#pragma unroll 2
  for (int i = 0; i < D / 16; ++i) {
    uint32_t hi[4], lo[4];
    float xs[16];
    if (p != nullptr) {
      load_q8(p + 16 * i, vec, xs);
      load_q8(p + 16 * i + 8, vec, xs + 8);
    } else {
#pragma unroll
      for (int j = 0; j < 16; ++j) xs[j] = 0.0f;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float y[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] = __fmul_rn(xs[4 * j + e], f);
      const uint32_t h0 = e4m3x2(y[0], y[1]), h1 = e4m3x2(y[2], y[3]);
      const uint32_t w0 = e4m3x2_half2(h0), w1 = e4m3x2_half2(h1);
      const float2 b0 = __half22float2(*reinterpret_cast<const __half2*>(&w0));
      const float2 b1 = __half22float2(*reinterpret_cast<const __half2*>(&w1));
      hi[j] = h0 | (h1 << 16);
      lo[j] = e4m3x2(__fsub_rn(y[0], b0.x), __fsub_rn(y[1], b0.y)) |
              (e4m3x2(__fsub_rn(y[2], b1.x), __fsub_rn(y[3], b1.y)) << 16);
    }
    *reinterpret_cast<uint4*>(&sm.q[t][0][i][r][0]) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
    *reinterpret_cast<uint4*>(&sm.q[t][1][i][r][0]) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
  }
  return amax < INFINITY ? fabsf(a.score_mul) * pow2f(-up) : __int_as_float(0x7FC00000);
}

template <int D>
__device__ void softmax_role(const AttnArgs& a, Walk w, Smem<D>& sm, const Ctx& x) {
  const KvArgs& c = a.c;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int t = warp >> 2, r = threadIdx.x & 127;
  const uint32_t lane_base = (uint32_t)(32 * (warp & 3)) << 16;
  const uint32_t ts = sm.tmem + t * BN + lane_base, to = sm.tmem + 2 * BN + t * D + lane_base;
  const float nan = __int_as_float(0x7FC00000);
  uint32_t ns = 0, no = 0, ng = 0;
  for (; w.more();) {
    const Segment sg = w.segment(a);
    const KvSeq s = w.s;
    if (sg.rows <= t * BM) {  // this tile has no row
      w.advance(a, sg);
      continue;
    }
    const int32_t* table = c.table + (int64_t)w.b * c.table_stride;
    const int row = w.t * kRows + t * BM + r;
    const bool have = t * BM + r < sg.rows;
    const int tok = row / c.group, head = sg.h * c.group + row % c.group;
    const float rm = stage_q<D>(a, sm, t, r, have ? static_cast<const __nv_bfloat16*>(a.q.p) + (int64_t)(s.first + tok) * a.q.ts +
                                                        (int64_t)head * a.q.hs : nullptr);
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    mbar_arrive(&sm.q_full[t]);
    const int lim = !have ? INT32_MAX : (a.causal ? s.kv - s.n + tok : s.kv - 1);
    int lim_min = lim;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) lim_min = min(lim_min, __shfl_xor_sync(0xffffffffu, lim_min, o));

    float m = -INFINITY, l = 0.0f;
    Groups g = load_groups(c, table, s.kv, sg.h, sg.blk0);
    for (int blk = sg.blk0; blk < sg.blk1; ++blk) {
      const Groups cur = g;
      if (blk + 1 < sg.blk1) g = load_groups(c, table, s.kv, sg.h, blk + 1);
      const bool masked = blk * BN + BN - 1 > lim_min || __any_sync(0xffffffffu, lane < 8 && cur.have < 16);
      const int col = lim == INT32_MAX ? BN : lim - blk * BN;  // last column this row sees
      // lane i < 8: the scale of group i's keys, the exponent and unscaling of its values
      const float gk = cur.ek == kExpNan ? nan : pow2f(cur.ek);
      const float ge = cur.ev == kExpNan ? nan : (float)cur.ev;
      const float gu = cur.ev == kExpNan ? nan : pow2f(-cur.ev);
      if (!wait_warp(x, &sm.s_full[t], ns++ & 1)) return;
      tc_fence_after();

      // ---- maximum
      float mx = -INFINITY;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        float v[32];
        tmem_ld16(ts + 32 * q, v);
        tmem_ld16(ts + 32 * q + 16, v + 16);
        tmem_wait_ld(v);
        tmem_tie(v + 16);
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
          const int gi = 2 * q + hf;
          const float k = __fmul_rn(rm, __shfl_sync(0xffffffffu, gk, gi)), e = __shfl_sync(0xffffffffu, ge, gi);
          float raw = -INFINITY;
          if (masked) {
            const int lc = min(col, 16 * gi + __shfl_sync(0xffffffffu, cur.have, gi) - 1);
#pragma unroll
            for (int j = 0; j < 16; ++j) raw = 16 * gi + j <= lc ? fmaxf(raw, v[16 * hf + j]) : raw;
          } else {
#pragma unroll
            for (int j = 0; j < 16; ++j) raw = fmaxf(raw, v[16 * hf + j]);
          }
          mx = fmaxf(mx, __fmaf_rn(raw, k, e));
        }
      }

      // ---- running maximum; O and l follow when it grew by more than 2^kGrow
      const bool grow = mx > __fadd_rn(m, kGrow);
      if (__any_sync(0xffffffffu, grow)) {
        const float mn = grow ? mx : m;
        const float f = mn == -INFINITY ? 1.0f : ex2(__fsub_rn(m, mn));
        l = __fmul_rn(l, f);
        m = mn;
        if (blk > sg.blk0) {
#pragma unroll
          for (int q = 0; q < D / 32; ++q) {
            float v[32];
            tmem_ld16(to + 32 * q, v);
            tmem_ld16(to + 32 * q + 16, v + 16);
            tmem_wait_ld(v);
            tmem_tie(v + 16);
            uint32_t b[32];
#pragma unroll
            for (int j = 0; j < 32; ++j) b[j] = __float_as_uint(__fmul_rn(v[j], f));
            tmem_st16(to + 32 * q, b);
            tmem_st16(to + 32 * q + 16, b + 16);
          }
        }
      }
      const float off = kPBits - (m == -INFINITY ? 0.0f : m);

      // ---- weights
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        float v[32];
        tmem_ld16(ts + 32 * q, v);
        tmem_ld16(ts + 32 * q + 16, v + 16);
        tmem_wait_ld(v);
        tmem_tie(v + 16);
        uint32_t b[16];
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
          const int gi = 2 * q + hf;
          const float k = __fmul_rn(rm, __shfl_sync(0xffffffffu, gk, gi));
          const float e = __fadd_rn(__shfl_sync(0xffffffffu, ge, gi), off);
          const float un = __shfl_sync(0xffffffffu, gu, gi);
          const int lc = min(col, 16 * gi + __shfl_sync(0xffffffffu, cur.have, gi) - 1);
          float2 sum = make_float2(0.0f, 0.0f);
#pragma unroll
          for (int j = 0; j < 16; j += 2) {
            const float2 y = __ffma2_rn(make_float2(v[16 * hf + j], v[16 * hf + j + 1]), make_float2(k, k), make_float2(e, e));
            float2 p = make_float2(ex2(y.x), ex2(y.y));
            if (masked) {
              p.x = 16 * gi + j <= lc ? p.x : 0.0f;
              p.y = 16 * gi + j + 1 <= lc ? p.y : 0.0f;
            }
            sum = __fadd2_rn(sum, p);
            const __half2 hp = __floats2half2_rn(p.x, p.y);
            b[8 * hf + j / 2] = *reinterpret_cast<const uint32_t*>(&hp);
          }
          const float sg1 = __fadd_rn(sum.x, sum.y);
          l = sg1 == 0.0f ? l : __fmaf_rn(sg1, un, l);
        }
        tmem_st16(ts + 16 * q, b);  // P over columns of S already read
      }
      st_wait();
      tc_fence_before();
      mbar_arrive(&sm.p_full[t]);
    }

    // ---- the tile's result
    if (!wait_warp(x, &sm.o_full[t], no++ & 1)) return;
    tc_fence_after();
    float* slot = partial_slot(a, blockIdx.x, sg.c0) + (int64_t)t * BM * (D + 2) + r;
    __nv_bfloat16* op = static_cast<__nv_bfloat16*>(a.out.p) + (int64_t)(s.first + tok) * a.out.ts + (int64_t)head * a.out.hs;
    auto put = [&](int d, const float* o, float inv) {  // 8 dims of a finished row
      uint32_t b[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const __nv_bfloat162 hb = __floats2bfloat162_rn(__fmul_rn(o[2 * j], inv), __fmul_rn(o[2 * j + 1], inv));
        b[j] = *reinterpret_cast<const uint32_t*>(&hb);
      }
      if (reinterpret_cast<uintptr_t>(op) % 16 == 0) {
        *reinterpret_cast<uint4*>(op + d) = make_uint4(b[0], b[1], b[2], b[3]);
      } else {
        uint16_t* o16 = reinterpret_cast<uint16_t*>(op + d);
#pragma unroll
        for (int j = 0; j < 8; ++j) o16[j] = (uint16_t)(b[j >> 1] >> (16 * (j & 1)));
      }
    };
    auto put_lse = [&](float mm, float ll) {
      if (a.lse) a.lse[(int64_t)(s.first + tok) * c.n_heads + head] = ll == 0.0f ? -INFINITY : (mm - kPBits + log2f(ll)) * kLn2;
    };
    const float inv = l == 0.0f ? 0.0f : __frcp_rn(l);
#pragma unroll
    for (int q = 0; q < D / 32; ++q) {
      float v[32];
      tmem_ld16(to + 32 * q, v);
      tmem_ld16(to + 32 * q + 16, v + 16);
      tmem_wait_ld(v);
      tmem_tie(v + 16);
      if (have && sg.whole) {
#pragma unroll
        for (int j = 0; j < 4; ++j) put(32 * q + 8 * j, v + 8 * j, inv);
      } else if (have) {
#pragma unroll
        for (int j = 0; j < 32; ++j) slot[(32 * q + j) * BM] = v[j];
      }
    }
    tc_fence_before();
    if (sg.whole) {
      if (have) put_lse(m, l);
    } else {
      if (have) {
        slot[D * BM] = m;
        slot[(D + 1) * BM] = l;
      }
      __threadfence();
      mbar_arrive(&sm.group[t]);
      if (!wait_warp(x, &sm.group[t], ng++ & 1)) return;
      if (r == 0) {
        int* arr = a.arrived + 2 * sg.c0 + t;
        const int last = atomicAdd(arr, 1) == sg.c1 - sg.c0;
        if (last) *arr = 0;  // as every call leaves it
        *(volatile int*)&sm.last[t] = last;
        __threadfence();
      }
      mbar_arrive(&sm.group[t]);
      if (!wait_warp(x, &sm.group[t], ng++ & 1)) return;
      if (*(volatile int*)&sm.last[t] && have) {
        __threadfence();
        const int64_t at = (int64_t)t * BM * (D + 2) + r;
        float mm = -INFINITY;
        for (int k = sg.c0; k <= sg.c1; ++k) mm = fmaxf(mm, __ldcg(partial_slot(a, k, sg.c0) + at + D * BM));
        const float base = mm == -INFINITY ? 0.0f : mm;
        float ll = 0.0f;
        for (int k = sg.c0; k <= sg.c1; ++k) {
          const float* sp = partial_slot(a, k, sg.c0) + at;
          ll = __fmaf_rn(__ldcg(sp + (D + 1) * BM), ex2(__fsub_rn(__ldcg(sp + D * BM), base)), ll);
        }
        const float iv = ll == 0.0f ? 0.0f : __frcp_rn(ll);
        for (int d = 0; d < D; d += 8) {
          float o[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) o[j] = 0.0f;
          for (int k = sg.c0; k <= sg.c1; ++k) {
            const float* sp = partial_slot(a, k, sg.c0) + at;
            const float f = ex2(__fsub_rn(__ldcg(sp + D * BM), base));
#pragma unroll
            for (int j = 0; j < 8; ++j) o[j] = __fmaf_rn(__ldcg(sp + (d + j) * BM), f, o[j]);
          }
          put(d, o, iv);
        }
        put_lse(mm, ll);
      }
    }
    w.advance(a, sg);
  }
}

template <int D>
__global__ void __launch_bounds__(kThreads, 1) paged_tiles_kernel(const __grid_constant__ AttnArgs a) {
  extern __shared__ unsigned char smem_raw[];
  Smem<D>& sm = *reinterpret_cast<Smem<D>*>(smem_raw + ((1024u - (smem_addr(smem_raw) & 1023u)) & 1023u));
  Walk w;
  if (!w.start(a)) return;
  const int warp = threadIdx.x >> 5;
  if (warp == kLoadWarp) {
    if ((threadIdx.x & 31) == 0) {
      for (int i = 0; i < NK; ++i) mbar_init(&sm.k_full[i], 1), mbar_init(&sm.k_empty[i], 1);
      for (int i = 0; i < NV; ++i) mbar_init(&sm.v_full[i], 1), mbar_init(&sm.v_empty[i], 128);
      for (int i = 0; i < NW; ++i) mbar_init(&sm.w_full[i], 128), mbar_init(&sm.w_empty[i], 1);
      for (int i = 0; i < 2; ++i) {
        mbar_init(&sm.q_full[i], 128);
        mbar_init(&sm.s_full[i], 1);
        mbar_init(&sm.p_full[i], 128);
        mbar_init(&sm.o_full[i], 1);
        mbar_init(&sm.group[i], 128);
      }
      mbar_init(&sm.drain, 1);
      sm.dead = 0;
      asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncwarp();
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&sm.tmem)),
                 "r"(kTmemCols)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    tc_fence_before();
  }
  __syncthreads();
  tc_fence_after();
  const Ctx x{a.wait_ns, a.c.status, &sm.dead};
  if (warp < 8) {
    softmax_role<D>(a, w, sm, x);
  } else if (warp < kMmaWarp) {
    widen_role<D>(a, w, sm, x);
  } else if (warp == kMmaWarp) {
    if ((threadIdx.x & 31) == 0) mma_role<D>(a, w, sm, x);
    __syncwarp();
  } else {
    load_role<D>(a, w, sm, x);
  }
  tc_fence_before();
  __syncthreads();
  if (warp == kLoadWarp) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(sm.tmem), "r"(kTmemCols) : "memory");
  }
}

template <int D>
cudaError_t launch(const AttnArgs& a, int64_t max_blocks, cudaStream_t st) {
  constexpr int kSmem = (int)sizeof(Smem<D>) + 1024;
  static_assert(kSmem <= 227 * 1024, "shared memory of a block");
  const cudaError_t e = cudaFuncSetAttribute(paged_tiles_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
  if (e != cudaSuccess) return e;
  AttnArgs b = a;
  b.min_units = 1;
  int64_t grid = kMaxTileBlocks;
  const int64_t most = tiles_upper(a.c, kRows) * a.c.kv_heads * max_blocks;
  if (grid > most) grid = most;
  paged_tiles_kernel<D><<<(unsigned)grid, kThreads, kSmem, st>>>(b);
  note_launches(1);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_paged_tiles(const AttnArgs& a, int head_dim, int max_kv, cudaStream_t st) {
  const int64_t mb = max_kv > BN ? ((int64_t)max_kv + BN - 1) / BN : 1;
  return head_dim == 128 ? launch<128>(a, mb, st) : launch<64>(a, mb, st);
}

}  // namespace awsrc
