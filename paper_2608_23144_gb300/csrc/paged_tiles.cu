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
//           a power of two per row to a largest element in [2^7, 2^8), is split into
//           an e4m3 term and an e5m2 one (two 8-bit products cost what one 16-bit
//           product costs; no key is ever converted). Beside the 4 bits of the first
//           a bf16 leaves at most 8 signed units, which e5m2 holds: elements from 2^-6
//           on are exact, smaller ones, whose first term is subnormal, within 2^-14
//           (all bf16 values tried). Of a row's largest element that is 2^-13 and
//           2^-21. An e4m3 second term ended at 2^-9: it lost bits from 2^-9 of the
//           largest element down and kept 2^-17. q in binary16 beside keys widened
//           like the values would be exact to 2^-39, and took 7% (four prompts) to
//           16% (chunks) longer: the widened keys' stores compete with the products
//           for shared memory;
//   p . V   kind::f16 with p in binary16 (from tensor memory: 11 bits, or 2^-25 under
//           a largest p of 2^6 or more; l takes it unrounded) and the value
//           codes widened to binary16, exactly, by four warps. Splitting p into
//           8-bit terms instead would cost the softmax warps two more
//           conversions per weight, five times the widening's instructions.
// Floor: 4 D flop per (row, token) at the bf16 rate.
//
// One thread block per SM and 256 rows (query tokens x the heads of a kv head)
// in two tiles of 128, so that one tile's softmax runs under the other's
// products. Warps 0-3 and 4-7: softmax, one row per thread; 8-11: widening; 12
// and 13: MMA issue; 14: bulk copies; 15: the walk over the share. Tensor memory:
// S 2 x 128 columns, over whose first 64 P is written; O 2 x D columns. Per tile
// and block of 128 tokens:
//   MMA:     P ready -> O += P V; S = Q K of the next block -> commit
//   softmax: S ready -> m, P, l; O rescaled by its own threads, only when a row
//            grew by more than 2^8 (the commit that made S ready also covers
//            the products that wrote O).
// The byte order of keys and values in the cache is the operand order the
// tensor cores read, so copies need no rearrangement.
//
// Work is shared out as in paged_attn.cu (UnitWalk). Tiles that thread blocks
// share leave partial results, which a second launch joins on the whole GPU:
// joined by the last block to arrive, the five parts of a tile took 60 us.
//
// Measured: four chunks of 1024 tokens on contexts of 20k beside decoding users (40
// heads, 8 kv heads) in 463 us, 1195 TFLOP/s or 63% of a large bf16 product; four
// prompts of up to 4096 tokens (28 heads, 4 kv heads) in 316 us, 796 TFLOP/s, the
// masked halves of diagonal blocks not counted. Bound: a block's 16 products of a
// tile take 1028 cycles by themselves (and 74 to commit) but about 1500 here, since
// q . k reads both operands from shared memory at its full rate, 128 bytes per
// cycle, beside the widening and the copies; a tile's softmax takes 1500 more before
// its next products can start. Two warps per softmax row (half the columns each)
// took 530 us for the chunks, as they get in the other tile's way.
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
constexpr int kThreads = 512;
constexpr int kMmaWarp = 12, kLoadWarp = 14;  // 15 walks the share
constexpr int kRing = 4, kReaders = 15;  // segments handed out ahead; warps that read them
constexpr int NK = 3, NV = 2, NW = 2;  // stages: keys, value codes, widened values
constexpr uint32_t kTmemCols = 512;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kPBits = 6.0f;         // p is at most 2^6 when m is the maximum,
constexpr float kTiny = 0x1p-80f;      // least score multiplier: times a block's scale, hidden scores of -inf stay -inf
constexpr float kGrow = 8.0f;          // and at most 2^(6 + 8) < 65504 when m lags
constexpr int kOver = 6;               // a tile's start and end and its masked blocks, in blocks (four prompts: 2: 423 us, 4: 330, 6: 321, 8: 337)
using Walk = UnitWalk<kRows, BN, 4, kOver>;

template <int N>
struct Idesc { static constexpr uint32_t value = idesc_f16(BM, N); };  // formats 0: e4m3, binary16
constexpr uint32_t kIdescAE5M2 = 1u << 7;  // format 1 of A in kind::f8f6f4

template <int D>
struct Smem {
  uint8_t q[2][2][D / 16][BM + 1][16];  // tile, term (e4m3, e5m2), 16 dims; runs one row apart in the banks
  uint8_t k[NK][D / 16][BN][16];
  uint8_t v[NV][BN / 16][D][16];
  uint8_t w[NW][BN / 8][D][16];     // binary16, 8 tokens
  unsigned long long k_full[NK], k_empty[NK], v_full[NV], v_empty[NV], w_full[NW], w_empty[NW];
  unsigned long long q_full[2], s_full[2], p_full[2], o_full[2], turn[2], drain[2];
  unsigned long long seg_full[kRing], seg_empty[kRing];
  SegRec seg[kRing];
  float4 group_of[8][2][8];  // softmax warp, block parity: scale of the keys, exponent and unscaling of the values, -
  uint8_t bad[kRows];        // the row sees marked values
  uint32_t tmem;
  int dead;
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

// D(tmem) (+)= A(smem, e4m3 or e5m2) B(smem, e4m3), 32 deep.
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
__device__ __forceinline__ float max3(float a, float b, float c) {  // one instruction of the half-rate pipe for two
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
__device__ __forceinline__ float max16(const float* v) {
  const float a = max3(v[0], v[1], v[2]), b = max3(v[3], v[4], v[5]), c = max3(v[6], v[7], v[8]);
  const float d = max3(v[9], v[10], v[11]), e = max3(v[12], v[13], v[14]);
  return max3(max3(a, b, c), d, fmaxf(e, v[15]));
}
__device__ __forceinline__ void st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// What the lanes of a warp know about the eight 16-token groups of a block,
// lane i < 8 about group i: tokens in it (0 for a page that cannot be right)
// and the exponents of its page.
struct Groups {
  int have, ek, ev;
};
__device__ __forceinline__ Groups load_groups(const KvArgs& c, const int32_t* table, int kv, int h, int blk) {
  const int lane = threadIdx.x & 31;
  const int j = blk * BN + 16 * (lane & 7);
  Groups g{0, 0, 0};
  if (lane < 8 && j < kv) {
    const int pg = table[j >> c.log_page];
    if (pg >= 0 && pg < c.n_pages) {
      g.have = min(16, kv - j);
      g.ek = __ldcg(c.k_exp + (int64_t)pg * c.kv_heads + h);
      g.ev = __ldcg(c.v_exp + (int64_t)pg * c.kv_heads + h);
    }
  }
  return g;
}

// The tokens of group lane % 8 alone.
__device__ __forceinline__ int group_tokens(const KvArgs& c, const int32_t* table, int kv, int blk) {
  const int j = blk * BN + 16 * (threadIdx.x & 7);
  if (j >= kv) return 0;
  const int pg = table[j >> c.log_page];
  return pg >= 0 && pg < c.n_pages ? min(16, kv - j) : 0;
}

// --------------------------------------------------------------------- walk --
// One lane walks the share and hands the segments to the roles through a ring,
// so that the walk's divisions are in one place and in nobody's way.
template <int D>
__device__ __noinline__ void walk_role(const AttnArgs& a, Walk w, Smem<D>& sm, const Ctx& x) {
  uint32_t i = 0;
  SharedTile mine{};
  a.shared[blockIdx.x] = mine;  // what stands there if a wait gives up
  for (; w.more();) {
    const Segment g = w.segment(a);
    if (!g.empty && !g.whole && g.c0 == (int)blockIdx.x)
      mine = SharedTile{w.t * kRows, g.rows, w.s.first, g.h, g.c1, {0, 0, 0}};
    if (!g.empty) {
      if (!wait_lane(x, &sm.seg_empty[i % kRing], ((i / kRing) & 1) ^ 1)) return;
      sm.seg[i % kRing] = w.record(g);
      mbar_arrive(&sm.seg_full[i % kRing]);
      ++i;
    }
    w.advance(a, g);
  }
  a.shared[blockIdx.x] = mine;
  if (!wait_lane(x, &sm.seg_empty[i % kRing], ((i / kRing) & 1) ^ 1)) return;
  sm.seg[i % kRing].b = -1;
  mbar_arrive(&sm.seg_full[i % kRing]);
}

// ------------------------------------------------------------------- copies --
template <int D>
__device__ void load_role(const AttnArgs& a, Smem<D>& sm, const Ctx& x) {
  const KvArgs& c = a.c;
  const int lane = threadIdx.x & 31;
  const int per = BN >> c.log_page;  // pages of a block
  const bool small = small_pages(c);
  uint32_t n = 0, is = 0;
  bool ok = true;
  for (; ok; ++is) {
    if (!(ok = wait_warp(x, &sm.seg_full[is % kRing], (is / kRing) & 1))) break;
    const SegRec& sg = sm.seg[is % kRing];
    if (sg.b < 0) break;
    const int32_t* table = c.table + (int64_t)sg.b * c.table_stride;
    // the softmax warps stage the segment's query rows some blocks from now
    const RowMap map(c, sg.row0);
    for (int r = lane; r < sg.rows; r += 32) {
      int tok, head;
      map.at(r, &tok, &head);
      const char* p = reinterpret_cast<const char*>(static_cast<const __nv_bfloat16*>(a.q.p) + (int64_t)(sg.first + tok) * a.q.ts +
                                                    (int64_t)(sg.h * c.group + head) * a.q.hs);
#pragma unroll
      for (int i = 0; i < 2 * D; i += 128) asm volatile("prefetch.global.L2 [%0];" ::"l"(p + i));
    }
    for (int blk = sg.blk0; ok && blk < sg.blk1; ++blk, ++n) {
      if ((int)n == a.stall) {  // the limit's test
        ok = false;
        break;
      }
      // lane i < per: page i of the block
      int pg = -1;
      const int j = blk * BN + (lane << c.log_page);
      if (lane < per && j < sg.kv) {
        pg = table[j >> c.log_page];
        if (pg < 0 || pg >= c.n_pages) {
          atomicOr(c.status, kFaultBatch);
          pg = -1;
        }
      }
      const uint32_t bytes = (uint32_t)(__popc(__ballot_sync(0xffffffffu, pg >= 0)) * D) << c.log_page;
      const int ks = n % NK, vs = n % NV;
      if (!(ok = wait_warp(x, &sm.k_empty[ks], ((n / NK) & 1) ^ 1))) break;
      if (small) {
#pragma unroll
        for (int j = 0; j < BN / 32; ++j) {  // a page's run per half warp
          const int pp = __shfl_sync(0xffffffffu, pg, 2 * j + (lane >> 4));
          if (pp < 0) continue;
          const uint8_t* src = c.k + block_off<D>(c, pp, sg.h) + 16 * (lane & 15);
#pragma unroll
          for (int run = 0; run < D / 16; ++run) copy16(&sm.k[ks][run][32 * j + lane][0], src + 256 * run);
        }
        copies_arrive(&sm.k_full[ks]);
      } else {
        if (lane == 0) mbar_expect_tx(&sm.k_full[ks], bytes);
        __syncwarp();
        for (int i0 = 0; i0 < (D / 16) * per; i0 += 32) {
          const int i = i0 + lane, p = i & (per - 1), run = i / per;
          const int pp = __shfl_sync(0xffffffffu, pg, p);
          if (pp >= 0 && run < D / 16)
            bulk_g2s(&sm.k[ks][run][p << c.log_page][0], c.k + block_off<D>(c, pp, sg.h) + ((run << c.log_page) << 4),
                     16u << c.log_page, &sm.k_full[ks]);
        }
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
    __syncwarp();
    if (lane == 0) mbar_arrive(&sm.seg_empty[is % kRing]);
  }
  copies_wait();
  if (!ok && lane == 0) {  // copies in flight land before the block ends
    for (uint32_t j = n > NK ? n - NK : 0; j < n; ++j) (void)mbar_wait(&sm.k_full[j % NK], (j / NK) & 1, x.wait_ns);
    for (uint32_t j = n > NV ? n - NV : 0; j < n; ++j) (void)mbar_wait(&sm.v_full[j % NV], (j / NV) & 1, x.wait_ns);
  }
}

// ----------------------------------------------------------------- products --
// One warp issues the products of tile t, so that its waits pass under the other
// tile's products. The two take turns, a block's products at a time: left to
// interleave, both tiles' products ended together and so did their softmax.
// A commit costs the tensor cores 74 cycles (measured; the 16 products of a block
// take 1028), so there is one per block: weights handed over (p_full) say that the
// scores they came from, and all products issued before those, are done.
template <int D>
__device__ void mma_role(Smem<D>& sm, const Ctx& x, int t, bool small) {
  constexpr uint32_t kIdescS = Idesc<BN>::value, kIdescO = Idesc<D>::value;
  const uint32_t ts = sm.tmem + t * BN, to = sm.tmem + 2 * BN + t * D;
  const uint64_t q0 = desc(smem_addr(&sm.q[t][0][0][0][0]), (BM + 1) * 16);
  const uint64_t k0 = desc(smem_addr(&sm.k[0][0][0][0]), BN * 16);
  const uint64_t v0 = desc(smem_addr(&sm.w[0][0][0][0]), D * 16);
  uint32_t n = 0, nq = 0, np = 0, turns = 0, is = 0;
  // copies 16 bytes at a time are ordinary writes to shared memory
  auto async_fence = [] { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); };
  // tile 0 has the first turn
  auto my_turn = [&]() {
    const uint32_t k = turns++;
    return t == 0 ? k == 0 || wait_lane(x, &sm.turn[0], (k - 1) & 1) : wait_lane(x, &sm.turn[1], k & 1);
  };
  auto qk = [&](uint32_t blk) {
    const uint64_t kd = k0 + (uint64_t)(blk % NK) * (sizeof(sm.k[0]) >> 4);
#pragma unroll
    for (int s = 0; s < D / 16; ++s)  // both terms: 32 dims a step, 2 runs of 16 further each
      umma_f8(ts, q0 + s * (2 * (BM + 1) * 16 >> 4), kd + (s & (D / 32 - 1)) * (2 * BN * 16 >> 4),
              s < D / 32 ? kIdescS : kIdescS | kIdescAE5M2, s > 0);
    umma_commit(&sm.s_full[t]);
  };
  bool ok = true, held = false;  // held: the widened values of block n - 1 are not given back yet
  for (; ok; ++is) {
    if (!(ok = wait_lane(x, &sm.seg_full[is % kRing], (is / kRing) & 1))) break;
    const SegRec& sg = sm.seg[is % kRing];
    if (sg.b < 0) break;
    const int nb = sg.blk1 - sg.blk0;
    if (sg.rows <= t * BM) {  // no row in this tile: its blocks pass
      if (!(ok = my_turn())) break;
      if (held) umma_commit(&sm.w_empty[(n - 1) % NW]);
      held = false;
      mbar_arrive(&sm.turn[t ^ 1]);
      for (int i = 0; ok && i < nb; ++i, ++n) {
        if (!(ok = wait_lane(x, &sm.k_full[n % NK], (n / NK) & 1))) break;
        mbar_arrive(&sm.k_empty[n % NK]);
        if (!(ok = wait_lane(x, &sm.w_full[n % NW], (n / NW) & 1))) break;
        mbar_arrive(&sm.w_empty[n % NW]);
        if (!(ok = my_turn())) break;
        mbar_arrive(&sm.turn[t ^ 1]);
      }
    } else {
      if (!(ok = wait_lane(x, &sm.q_full[t], nq++ & 1)) || !(ok = wait_lane(x, &sm.k_full[n % NK], (n / NK) & 1)) || !(ok = my_turn()))
        break;
      tc_fence_after();
      if (small) async_fence();
      qk(n);
      mbar_arrive(&sm.turn[t ^ 1]);
      for (int i = 0; i < nb; ++i, ++n) {
        const uint32_t n1 = n + 1;
        if (i + 1 < nb && !(ok = wait_lane(x, &sm.k_full[n1 % NK], (n1 / NK) & 1))) break;
        if (!(ok = wait_lane(x, &sm.w_full[n % NW], (n / NW) & 1))) break;
        const uint64_t vd = v0 + (uint64_t)(n % NW) * (sizeof(sm.w[0]) >> 4);
        if (!(ok = wait_lane(x, &sm.p_full[t], np++ & 1))) break;
        mbar_arrive(&sm.k_empty[n % NK]);
        if (held) mbar_arrive(&sm.w_empty[(n - 1) % NW]);
        held = true;
        if (!(ok = my_turn())) break;
        tc_fence_after();
        if (small) async_fence();
#pragma unroll
        for (int s = 0; s < BN / 16; ++s)
          umma_f16_ts(to, ts + s * 8, vd + s * (2 * D * 16 >> 4), kIdescO, i + s > 0);
        if (i + 1 < nb)
          qk(n1);
        else
          umma_commit(&sm.o_full[t]);
        mbar_arrive(&sm.turn[t ^ 1]);
      }
    }
    mbar_arrive(&sm.seg_empty[is % kRing]);
  }
  if (!ok) {  // products in flight end before the block does
    umma_commit(&sm.drain[t]);
    (void)mbar_wait(&sm.drain[t], 0, x.wait_ns);
  }
}

// ----------------------------------------------------------------- widening --
template <int D>
__device__ void widen_role(const AttnArgs& a, Smem<D>& sm, const Ctx& x) {
  const KvArgs& c = a.c;
  const int tid = threadIdx.x & 127;
  uint32_t n = 0, is = 0;
  bool ok = true;
  for (; ok; ++is) {
    if (!(ok = wait_warp(x, &sm.seg_full[is % kRing], (is / kRing) & 1))) break;
    const SegRec& sg = sm.seg[is % kRing];
    if (sg.b < 0) break;
    const int32_t* table = c.table + (int64_t)sg.b * c.table_stride;
    int next = group_tokens(c, table, sg.kv, sg.blk0);
    for (int blk = sg.blk0; blk < sg.blk1; ++blk, ++n) {
      const int cur = next;
      if (blk + 1 < sg.blk1) next = group_tokens(c, table, sg.kv, blk + 1);
      // rows that hold no token may hold any bytes, e4m3's NaN among them: zeros
      const bool tail = __any_sync(0xffffffffu, cur < 16);
      if (!(ok = wait_warp(x, &sm.v_full[n % NV], (n / NV) & 1)) ||
          !(ok = wait_warp(x, &sm.w_empty[n % NW], ((n / NW) & 1) ^ 1)))
        break;
      const uint8_t* src = &sm.v[n % NV][0][0][0];
      uint8_t* dst = &sm.w[n % NW][0][0][0];
#pragma unroll 2
      for (int i = 0; i < BN / 16 * D / 128; ++i) {
        const int e = tid + 128 * i, run = e / D, d = e % D;
        uint4 v = *reinterpret_cast<const uint4*>(src + (size_t)e * 16);
        if (tail) {
          const int have = __shfl_sync(0xffffffffu, cur, run);
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
    __syncwarp();
    if ((tid & 31) == 0) mbar_arrive(&sm.seg_empty[is % kRing]);
  }
}

// ------------------------------------------------------------------ softmax --
__device__ __forceinline__ uint32_t e4m3x2_h(__half2 v) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f16x2 %0, %1;" : "=h"(r) : "r"(*reinterpret_cast<const uint32_t*>(&v)));
  return r;
}

__device__ __forceinline__ uint32_t e5m2x2_h(__half2 v) {
  uint16_t r;
  asm("cvt.rn.satfinite.e5m2x2.f16x2 %0, %1;" : "=h"(r) : "r"(*reinterpret_cast<const uint32_t*>(&v)));
  return r;
}

// The warp's 32 query rows of tile t -> two 8-bit terms in shared memory; returns
// the multiplier of the scores of row 32 (warp % 4) + lane. Consecutive lanes
// read consecutive dims of a row (8 each), loads of the next
// rows in flight.
template <int D>
__device__ __noinline__ float stage_q(const AttnArgs& a, Smem<D>& sm, int t, const SegRec& sg) {
  const RowMap map(a.c, sg.row0);
  const int h = sg.h, rows = sg.rows;
  constexpr int kLanes = D / 8, kPer = 32 / kLanes, kIt = 32 / kPer;  // lanes of a row, rows at a time
  constexpr int kB = 8;                                               // such steps worked on together
  const int lane = threadIdx.x & 31, r0 = threadIdx.x & 96;
  const int sub = lane % kLanes, first = t * BM + r0 + lane / kLanes;
  const int64_t ts = a.q.ts, hs = a.q.hs;
  const __nv_bfloat16* qp = static_cast<const __nv_bfloat16*>(a.q.p) + sg.first * ts + (int64_t)h * a.c.group * hs + 8 * sub;
  float rm = 0.0f;
#pragma unroll 1
  for (int i0 = 0; i0 < kIt; i0 += kB) {
    uint4 v[kB];
#pragma unroll
    for (int b = 0; b < kB; ++b) {
      int tok, head;  // rows past the last repeat it: no branch holds a load back
      map.at(min(first + kPer * (i0 + b), rows - 1), &tok, &head);
      v[b] = __ldcg(reinterpret_cast<const uint4*>(qp + tok * ts + head * hs));
    }
    uint32_t am[kB];  // largest magnitude, as bits: bf16 patterns order like their values, NaN above infinity
#pragma unroll
    for (int b = 0; b < kB; ++b) {
      const uint32_t x = __vmaxu2(__vmaxu2(v[b].x & 0x7FFF7FFFu, v[b].y & 0x7FFF7FFFu),
                                  __vmaxu2(v[b].z & 0x7FFF7FFFu, v[b].w & 0x7FFF7FFFu));
      am[b] = max(x & 0xFFFFu, x >> 16);
    }
#pragma unroll
    for (int o = 1; o < kLanes; o <<= 1)
#pragma unroll
      for (int b = 0; b < kB; ++b) am[b] = max(am[b], __shfl_xor_sync(0xffffffffu, am[b], o));
#pragma unroll
    for (int b = 0; b < kB; ++b) {
      // the row times 2^up has its largest element in [2^7, 2^8)
      const int up = min(max(7 - ((int)(am[b] >> 7) - 127), -120), 100);
      const float f = a.score_mul < 0.0f ? -pow2f(up) : pow2f(up);
      const float mul = am[b] < 0x7F80u ? fabsf(a.score_mul) * pow2f(-up) : __int_as_float(0x7FC00000);
      const float got = __shfl_sync(0xffffffffu, mul, (lane % kPer) * kLanes);
      if (lane / kPer == i0 + b) rm = got;
      const uint32_t w[4] = {v[b].x, v[b].y, v[b].z, v[b].w};
      uint32_t hi[4], lo[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        // binary16 holds the scaled values down to 2^-32 of the row's largest
        const __half2 y = __floats2half2_rn(__fmul_rn(__uint_as_float(w[j] << 16), f),
                                            __fmul_rn(__uint_as_float(w[j] & 0xFFFF0000u), f));
        hi[j] = e4m3x2_h(y);
        const uint32_t back = e4m3x2_half2(hi[j]);
        lo[j] = e5m2x2_h(__hsub2(y, *reinterpret_cast<const __half2*>(&back)));
      }
      const int r = r0 + kPer * (i0 + b) + lane / kLanes;
      *reinterpret_cast<uint2*>(&sm.q[t][0][sub >> 1][r][8 * (sub & 1)]) = make_uint2(hi[0] | hi[1] << 16, hi[2] | hi[3] << 16);
      *reinterpret_cast<uint2*>(&sm.q[t][1][sub >> 1][r][8 * (sub & 1)]) = make_uint2(lo[0] | lo[1] << 16, lo[2] | lo[3] << 16);
    }
  }
  return rm;
}

// 16 dims of a finished row.
__device__ __forceinline__ void put16(__nv_bfloat16* p, const float* o, float inv) {
  uint32_t b[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const __nv_bfloat162 hb = __floats2bfloat162_rn(__fmul_rn(o[2 * j], inv), __fmul_rn(o[2 * j + 1], inv));
    b[j] = *reinterpret_cast<const uint32_t*>(&hb);
  }
  if (reinterpret_cast<uintptr_t>(p) % 32 == 0) {  // a whole sector
    asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "r"(b[0]), "r"(b[1]), "r"(b[2]), "r"(b[3]),
                 "r"(b[4]), "r"(b[5]), "r"(b[6]), "r"(b[7])
                 : "memory");
  } else {
    *reinterpret_cast<uint4*>(p) = make_uint4(b[0], b[1], b[2], b[3]);
    *reinterpret_cast<uint4*>(p + 8) = make_uint4(b[4], b[5], b[6], b[7]);
  }
}

__device__ __forceinline__ float lse_of(float m, float l) {
  return l == 0.0f ? -INFINITY : (m - kPBits + log2f(l)) * kLn2;
}

// The result of a tile: its rows out, or a partial result. False when a wait
// gave up.
template <int D>
__device__ __noinline__ bool finish_tile(const AttnArgs& a, Smem<D>& sm, const Ctx& x, int t, const SegRec& cs, float m,
                                         float l, uint32_t no) {
  const KvArgs& c = a.c;
  const int r = threadIdx.x & 127;
  const uint32_t to = sm.tmem + 2 * BN + t * D + ((uint32_t)(32 * ((threadIdx.x >> 5) & 3)) << 16);
  const bool have = t * BM + r < cs.rows;
  int tok, head;
  RowMap(c, cs.row0).at(t * BM + r, &tok, &head);
  head += cs.h * c.group;
  // ---- the tile's result
  if (!wait_warp(x, &sm.o_full[t], no & 1)) return false;
  tc_fence_after();
  float* slot = partial_slot(a, blockIdx.x, cs.c0) + (int64_t)t * BM * (D + 2) + r;
  __nv_bfloat16* op = static_cast<__nv_bfloat16*>(a.out.p) + (int64_t)(cs.first + tok) * a.out.ts + (int64_t)head * a.out.hs;
  const float nan = __int_as_float(0x7FC00000);
  const bool bad = sm.bad[t * BM + r];
  const float inv = bad ? nan : (l == 0.0f ? 0.0f : __frcp_rn(l));
#pragma unroll 1
  for (int q = 0; q < D / 16; ++q) {
    float v[16];
    tmem_ld16(to + 16 * q, v);
    tmem_wait_ld(v);
    if (have && cs.whole) {
      put16(op + 16 * q, v, inv);
    } else if (have) {
#pragma unroll
      for (int j = 0; j < 16; ++j) slot[(16 * q + j) * BM] = v[j];
    }
  }
  tc_fence_before();
  if (!have) return true;
  if (cs.whole) {
    if (a.lse) a.lse[(int64_t)(cs.first + tok) * c.n_heads + head] = lse_of(m, l);
  } else {
    slot[D * BM] = m;
    slot[(D + 1) * BM] = l;
    if (bad) {
#pragma unroll 1
      for (int d = 0; d < D; ++d) slot[d * BM] = nan;
    }
  }
  return true;
}

template <int D>
__device__ void softmax_role(const AttnArgs& a, Smem<D>& sm, const Ctx& x) {
  const KvArgs& c = a.c;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int t = warp >> 2, r = threadIdx.x & 127;
  const uint32_t lane_base = (uint32_t)(32 * (warp & 3)) << 16;
  const uint32_t ts = sm.tmem + t * BN + lane_base, to = sm.tmem + 2 * BN + t * D + lane_base;
  const float nan = __int_as_float(0x7FC00000);
  uint32_t ns = 0, no = 0;
  // The ring slot of the next segment with rows of this tile, its query rows sent
  // to the MMAs; kEnd, kGone when a wait gave up, or kLater: while a slot is held
  // no segment is passed over, or the ring could run full of what is held.
  constexpr int kEnd = -1, kGone = -2, kLater = -3;
  uint32_t is = 0;
  float rm = 0.0f;
  auto next = [&](bool held) -> int {
    for (;; ++is) {
      const uint32_t slot = is % kRing;
      if (!wait_warp(x, &sm.seg_full[slot], (is / kRing) & 1)) return kGone;
      if (sm.seg[slot].b < 0) return kEnd;
      if (sm.seg[slot].rows > t * BM) {
        rm = stage_q<D>(a, sm, t, sm.seg[slot]);
        rm = rm < kTiny ? kTiny : rm;
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        mbar_arrive(&sm.q_full[t]);
        ++is;
        return (int)slot;
      }
      if (held) return kLater;
      __syncwarp();
      if (lane == 0) mbar_arrive(&sm.seg_empty[slot]);
    }
  };
  for (int slot = next(false); slot >= 0;) {
    const SegRec& cs = sm.seg[slot];
    const int32_t* table = c.table + (int64_t)cs.b * c.table_stride;
    const int kv = cs.kv, blk1 = cs.blk1, h = cs.h;
    int lim = INT32_MAX;  // last token this row sees
    if (t * BM + r < cs.rows) {
      int tok, head;
      RowMap(c, cs.row0).at(t * BM + r, &tok, &head);
      lim = a.causal ? kv - cs.n + tok : kv - 1;
    }
    int lim_min = lim;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) lim_min = min(lim_min, __shfl_xor_sync(0xffffffffu, lim_min, o));
    float m = -INFINITY, l = 0.0f;
    sm.bad[threadIdx.x] = 0;
    Groups g = load_groups(c, table, kv, h, cs.blk0);
    for (int blk = cs.blk0; blk < blk1; ++blk) {
      const Groups cur = g;
      if (blk + 1 < blk1) g = load_groups(c, table, kv, h, blk + 1);
      // lane i < 8: the scale of group i's keys, the exponent and unscaling of its values, its tokens
      const bool mark = cur.ek == kExpNan, mark_v = cur.ev == kExpNan;
      const bool odd = __any_sync(0xffffffffu, lane < 8 && (cur.have < 16 || mark || mark_v));
      const bool masked = blk * BN + BN - 1 > lim_min || odd;
      if (odd) {  // marked values: O will be NaN for the rows that see one, the scores and l are what they are
        const uint32_t groups = __ballot_sync(0xffffffffu, mark_v);
        if (groups && lim >= blk * BN + 16 * (__ffs(groups) - 1)) sm.bad[threadIdx.x] = 1;
      }
      float4* gc = sm.group_of[warp][blk & 1];
      if (lane < 8)
        gc[lane] = make_float4(mark ? 1.0f : pow2f(cur.ek), mark_v ? 0.0f : (float)cur.ev, mark_v ? 1.0f : pow2f(-cur.ev), 0.0f);
      __syncwarp();
      if (!wait_warp(x, &sm.s_full[t], ns++ & 1)) return;
      tc_fence_after();
      if (masked) {  // hidden tokens to -inf, visible ones of marked keys to NaN, in place
        const int col = lim == INT32_MAX ? BN : lim - blk * BN;  // last column this row sees
#pragma unroll 1
        for (int i = 0; i < 8; ++i) {
          float v[16];
          tmem_ld16(ts + 16 * i, v);
          tmem_wait_ld(v);
          const int lc = min(col - 16 * i, __shfl_sync(0xffffffffu, cur.have, i) - 1);
          const bool bad = __shfl_sync(0xffffffffu, mark, i);
          uint32_t u[16];
#pragma unroll
          for (int j = 0; j < 16; ++j) u[j] = __float_as_uint(j > lc ? -INFINITY : (bad ? nan : v[j]));
          tmem_st16(ts + 16 * i, u);
        }
        st_wait();
      }

      // ---- the block's maximum, columns 64 .. 127 first; 0 .. 63 stay in registers
      // for their weights. What a segment does once lives in functions of its own:
      // in line, the roles' code outgrew the instruction cache
      float mx = -INFINITY, v[64];
#pragma unroll
      for (int q = 4; q >= 0; q -= 4) {
#pragma unroll
        for (int i = 0; i < 4; ++i) tmem_ld16(ts + 16 * (q + i), v + 16 * i);
        tmem_wait_ld(v);
#pragma unroll
        for (int i = 1; i < 4; ++i) tmem_tie(v + 16 * i);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float4 k = gc[q + i];
          mx = fmaxf(mx, __fmaf_rn(max16(v + 16 * i), __fmul_rn(rm, k.x), k.y));
        }
      }

      // ---- running maximum; O and l follow when it grew by more than 2^kGrow
      const bool grow = mx > __fadd_rn(m, kGrow);
      if (__any_sync(0xffffffffu, grow)) {
        const float mn = grow ? mx : m;
        const float f = mn == -INFINITY ? 1.0f : ex2(__fsub_rn(m, mn));
        l = __fmul_rn(l, f);
        m = mn;
        if (blk > cs.blk0) {
#pragma unroll 1
          for (int q = 0; q < D / 16; ++q) {
            float o[16];
            tmem_ld16(to + 16 * q, o);
            tmem_wait_ld(o);
            uint32_t b[16];
#pragma unroll
            for (int j = 0; j < 16; ++j) b[j] = __float_as_uint(__fmul_rn(o[j], f));
            tmem_st16(to + 16 * q, b);
          }
        }
      }
      const float off = rm < INFINITY ? kPBits - (m == -INFINITY ? 0.0f : m) : nan;

      // ---- weights, P over columns of S already read
#pragma unroll
      for (int q = 0; q < 8; q += 4) {
        uint32_t u[32];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float4 k = gc[q + i];
          const float kx = __fmul_rn(rm, k.x), e = __fadd_rn(k.y, off);
          float2 p[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const float2 y = __ffma2_rn(make_float2(v[16 * i + 2 * j], v[16 * i + 2 * j + 1]), make_float2(kx, kx),
                                        make_float2(e, e));
            p[j] = make_float2(ex2(y.x), ex2(y.y));
            const __half2 hp = __floats2half2_rn(p[j].x, p[j].y);
            u[8 * i + j] = *reinterpret_cast<const uint32_t*>(&hp);
          }
          const float2 s0 = __fadd2_rn(__fadd2_rn(p[0], p[1]), __fadd2_rn(p[2], p[3]));
          const float2 s1 = __fadd2_rn(__fadd2_rn(p[4], p[5]), __fadd2_rn(p[6], p[7]));
          const float2 s2 = __fadd2_rn(s0, s1);
          l = __fmaf_rn(__fadd_rn(s2.x, s2.y), k.z, l);
        }
        if (q == 0) {
#pragma unroll
          for (int i = 0; i < 4; ++i) tmem_ld16(ts + 64 + 16 * i, v + 16 * i);
        }
        tmem_st16(ts + 8 * q, u);
        tmem_st16(ts + 8 * q + 16, u + 16);
        if (q == 0) {
          tmem_wait_ld(v);
#pragma unroll
          for (int i = 1; i < 4; ++i) tmem_tie(v + 16 * i);
        }
      }
      st_wait();
      tc_fence_before();
      mbar_arrive(&sm.p_full[t]);
    }
    // the last block's scores are done with the query staging: the next tile's
    // rows go there while this one's last products run
    int after = next(true);
    if (after == kGone || !finish_tile<D>(a, sm, x, t, cs, m, l, no++)) return;
    __syncwarp();
    if (lane == 0) mbar_arrive(&sm.seg_empty[slot]);
    if (after == kLater) after = next(false);
    slot = after;
  }
}

template <int D>
__global__ void __launch_bounds__(kThreads, 1) paged_tiles_kernel(const __grid_constant__ AttnArgs a) {
  extern __shared__ unsigned char smem_raw[];
  Smem<D>& sm = *reinterpret_cast<Smem<D>*>(smem_raw + ((1024u - (smem_addr(smem_raw) & 1023u)) & 1023u));
  wait_for_previous();
  let_next_start();
  Walk w;
  if (!w.start(a)) {
    if (threadIdx.x == 0) a.shared[blockIdx.x] = SharedTile{};
    return;
  }
  const int warp = threadIdx.x >> 5;
  if (warp == kLoadWarp) {
    if ((threadIdx.x & 31) == 0) {
      for (int i = 0; i < NK; ++i) mbar_init(&sm.k_full[i], small_pages(a.c) ? 32 : 1), mbar_init(&sm.k_empty[i], 2);
      for (int i = 0; i < NV; ++i) mbar_init(&sm.v_full[i], 1), mbar_init(&sm.v_empty[i], 128);
      for (int i = 0; i < NW; ++i) mbar_init(&sm.w_full[i], 128), mbar_init(&sm.w_empty[i], 2);
      for (int i = 0; i < 2; ++i) {
        mbar_init(&sm.q_full[i], 128);
        mbar_init(&sm.s_full[i], 1);
        mbar_init(&sm.p_full[i], 128);
        mbar_init(&sm.o_full[i], 1);
        mbar_init(&sm.turn[i], 1);
        mbar_init(&sm.drain[i], 1);
      }
      for (int i = 0; i < kRing; ++i) mbar_init(&sm.seg_full[i], 1), mbar_init(&sm.seg_empty[i], kReaders);
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
    softmax_role<D>(a, sm, x);
  } else {
    if (warp < kMmaWarp) {
      widen_role<D>(a, sm, x);
    } else if (warp < kLoadWarp) {
      if ((threadIdx.x & 31) == 0) mma_role<D>(sm, x, warp - kMmaWarp, small_pages(a.c));
    } else if (warp == kLoadWarp) {
      load_role<D>(a, sm, x);
    } else if ((threadIdx.x & 31) == 0) {
      walk_role<D>(a, w, sm, x);
    }
    __syncwarp();
  }
  tc_fence_before();
  __syncthreads();
  if (warp == kLoadWarp) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(sm.tmem), "r"(kTmemCols) : "memory");
  }
}

// Joins the parts of the shared tile that begins in block blockIdx.x's share: 32
// rows a block, a row per lane, D / 8 dims per warp; parts in order, four of them
// in flight. The rows leave through shared memory.
template <int D>
__global__ void __launch_bounds__(256) paged_join_kernel(const __grid_constant__ AttnArgs a) {
  constexpr int kD = D / 8;
  __shared__ float rows[32][D + 1];
  wait_for_previous();
  const SharedTile tile = a.shared[blockIdx.x];
  const int r0 = 32 * blockIdx.y;
  if (r0 >= tile.rows) return;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c0 = blockIdx.x;
  const int r = r0 + lane;
  const bool have = r < tile.rows;
  const int64_t at = (int64_t)(r / BM) * BM * (D + 2) + r % BM;
  float m = -INFINITY;
#pragma unroll 4
  for (int k = c0; k <= tile.c1; ++k) m = fmaxf(m, partial_slot(a, k, c0)[at + D * BM]);
  const float base = m == -INFINITY ? 0.0f : m;
  float l = 0.0f, o[kD];
#pragma unroll
  for (int j = 0; j < kD; ++j) o[j] = 0.0f;
#pragma unroll 4
  for (int k = c0; k <= tile.c1; ++k) {
    const float* sp = partial_slot(a, k, c0) + at;
    const float f = ex2(__fsub_rn(sp[D * BM], base));
    l = __fmaf_rn(sp[(D + 1) * BM], f, l);
#pragma unroll
    for (int j = 0; j < kD; ++j) o[j] = __fmaf_rn(sp[(kD * warp + j) * BM], f, o[j]);
  }
  const float inv = l == 0.0f ? 0.0f : __frcp_rn(l);
#pragma unroll
  for (int j = 0; j < kD; ++j) rows[lane][kD * warp + j] = __fmul_rn(o[j], inv);
  const RowMap map(a.c, tile.row0);
  if (warp == 0 && have && a.lse) {
    int tok, head;
    map.at(r, &tok, &head);
    a.lse[(int64_t)(tile.first + tok) * a.c.n_heads + tile.h * a.c.group + head] = lse_of(m, l);
  }
  __syncthreads();
  for (int i = threadIdx.x; i < 32 * D / 8; i += 256) {
    const int rr = i / (D / 8), d = i % (D / 8) * 8;
    if (r0 + rr >= tile.rows) break;
    int tok, head;
    map.at(r0 + rr, &tok, &head);
    uint32_t b[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const __nv_bfloat162 hb = __floats2bfloat162_rn(rows[rr][d + 2 * j], rows[rr][d + 2 * j + 1]);
      b[j] = *reinterpret_cast<const uint32_t*>(&hb);
    }
    *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(a.out.p) + (int64_t)(tile.first + tok) * a.out.ts +
                              (int64_t)(tile.h * a.c.group + head) * a.out.hs + d) = make_uint4(b[0], b[1], b[2], b[3]);
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
  const cudaError_t k = launch_next(paged_tiles_kernel<D>, dim3((unsigned)grid), kThreads, kSmem, b, st);
  if (k != cudaSuccess) return k;
  note_launches(1);
  if (grid > 1) {  // one block shares no tile
    const cudaError_t j = launch_next(paged_join_kernel<D>, dim3((unsigned)grid, kRows / 32), 256, 0, b, st);
    if (j != cudaSuccess) return j;
    note_launches(1);
  }
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_paged_tiles(const AttnArgs& a, int head_dim, int max_kv, cudaStream_t st) {
  const int64_t mb = max_kv > BN ? ((int64_t)max_kv + BN - 1) / BN : 1;
  return head_dim == 128 ? launch<128>(a, mb, st) : launch<64>(a, mb, st);
}

}  // namespace awsrc
