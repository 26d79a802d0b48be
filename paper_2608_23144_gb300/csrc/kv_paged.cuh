// kv_paged.cuh — what the paged-cache kernels share: the cache and batch as the
// kernels see them, per-sequence checks, byte offsets of the code layouts and
// e4m3 conversions.
#pragma once

#include <cuda_fp8.h>

#include "common.cuh"

namespace awsrc {

constexpr int kExpNan = -128;  // exponent of a block that received a non-finite value
constexpr int kExpMin = -32, kExpMax = 31;

struct KvRows {  // [token][head][dim], strides in elements
  void* p;
  int64_t ts, hs;
};

// Every row of r (elements of elt bytes) starts on a 16-byte boundary.
inline bool rows_aligned(const KvRows& r, size_t elt) {
  return (reinterpret_cast<uintptr_t>(r.p) | (uintptr_t)(r.ts * (int64_t)elt) | (uintptr_t)(r.hs * (int64_t)elt)) % 16 == 0;
}

struct KvArgs {
  uint8_t *k, *v;
  int8_t *k_exp, *v_exp;
  int n_pages, page, log_page, kv_heads;
  int n_heads, group;  // query heads, query heads per kv head
  int n_seq, n_tok, table_stride;
  const int32_t *q_start, *kv_len, *table;
  uint32_t* status;
};

// The new tokens of sequence b: rows [first, first + n) of q, the last n of its
// kv tokens. n = -1 for an entry that cannot be right.
struct KvSeq {
  int first, n, kv;
};

__device__ __forceinline__ KvSeq kv_seq(const KvArgs& a, int b) {
  const int q0 = a.q_start[b], q1 = a.q_start[b + 1], kv = a.kv_len[b];
  const bool ok = q0 >= 0 && q0 <= q1 && q1 <= a.n_tok && kv >= q1 - q0 &&
                  (int64_t)kv <= ((int64_t)a.table_stride << a.log_page);
  return KvSeq{q0, ok ? q1 - q0 : -1, ok ? kv : 0};
}

// Byte offset of the block (pg, head) in k or v: blocks are page * D bytes.
template <int D>
__device__ __forceinline__ int64_t block_off(const KvArgs& a, int pg, int head) {
  return (((int64_t)pg * a.kv_heads + head) * D) << a.log_page;
}

// Smallest e with amax <= 448 * 2^e (448 = 1.75 * 2^8), at least kExpMin;
// kExpNan for a NaN, an infinity or a value above 448 * 2^kExpMax.
__device__ __forceinline__ int block_exponent(float amax) {
  if (!(amax <= 448.0f * 0x1p31f)) return kExpNan;
  const uint32_t u = __float_as_uint(amax);
  const int e = (int)(u >> 23) - 127 - 8 + ((u & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  return max(e, kExpMin);  // zeros and subnormals too
}

// Two e4m3 codes of a (low byte) and b, to nearest even; |a|, |b| <= 448.
__device__ __forceinline__ uint32_t e4m3x2(float a, float b) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(b), "f"(a));
  return r;
}

// The values of two codes as binary16 (exact).
__device__ __forceinline__ uint32_t e4m3x2_half2(uint32_t codes) {
  uint32_t r;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"((uint16_t)codes));
  return r;
}

// Attention: thread blocks a launch may have (two per SM, four with 64-dim
// heads), each with two slots for partial results of the first and last tile it
// shares with others.
constexpr int max_attn_blocks(int dim) { return dim == 64 ? 608 : 304; }
constexpr int kSlotRows = 64;
// The tensor-memory kernel: one per SM, 256 rows.
constexpr int kMaxTileBlocks = 152;
constexpr int kTileSlotRows = 256;

struct AttnArgs {
  KvArgs c;
  KvRows q, out;
  float* lse;
  float score_mul;  // sm_scale log2(e)
  int causal, vec, vec_out;  // rows of q, of out are 16-byte aligned
  int min_units;    // least share of a block
  int* arrived;     // per block: arrivals at the shared tile that begins in its share (row kernel)
  struct SharedTile* shared;  // per block: the shared tile that begins in its share, when a second launch joins
  float* partial;
  int64_t slot_floats;
  uint64_t wait_ns;  // limit of the kernels' waits
  int stall;         // test of that limit: no copies from this block of tokens on (-1: never)
};

// ------------------------------------------------------------ work sharing --
// A batch is cut into units: (sequence, tile of ROWS query rows, kv head, block
// of UNIT tokens), in this order; rows are query tokens x the heads of a kv
// head. A tile has as many blocks as its last row sees tokens, at least one;
// OVER further units in front of them stand for what starting and finishing a
// tile costs (but not where shares are padded, below). The thread blocks of a launch take equal contiguous shares, a
// segment being the part of one (tile, head) in a share.
struct Segment {
  int h, blk0, blk1;  // kv head, blocks [blk0, blk1)
  int rows;           // query rows of the tile
  int64_t first;      // unit of block 0
  bool empty;         // no block of it lies in this share
  int c0, c1;         // thread blocks that share (tile, head)
  bool whole;         // this one has it alone
};

// A segment as the kernels pass it through shared memory: blocks [blk0, blk1) of
// kv head h for the query rows [row0, row0 + rows) of sequence b, whose new tokens
// are rows first .. first + n of q; b < 0 ends the walk.
struct SegRec {
  int b, h, blk0, blk1, row0, rows, first, n, kv, c0, c1, whole;
};

template <int ROWS, int UNIT, int WARPS, int OVER>
struct UnitWalk {
  int64_t chunk, u, u_end, tile_first;
  int b, t, blocks;  // sequence, tile and the tile's blocks
  int pad;           // a (tile, head) takes a multiple of this many units
  KvSeq s;

  __device__ __forceinline__ static int blocks_of(const AttnArgs& a, const KvSeq& s, int t) {
    int see = s.kv;
    if (a.causal) {
      const int last = min((t + 1) * ROWS, s.n * a.c.group) - 1;
      see = s.kv - s.n + last / a.c.group + 1;
    }
    return max(1, (see + UNIT - 1) / UNIT);
  }
  __device__ __forceinline__ static int tiles_of(const AttnArgs& a, const KvSeq& s) {
    return s.n > 0 ? (s.n * a.c.group + ROWS - 1) / ROWS : 0;
  }
  __device__ __forceinline__ static int span_of(int blocks, int pad) {
    return pad == 1 ? blocks + OVER : (blocks + pad - 1) / pad * pad;
  }
  __device__ __forceinline__ int lead() const { return pad == 1 ? OVER : 0; }  // units in front of block 0
  // Units of the tiles of s, or with `want` >= 0 the tile that holds unit `want`
  // of them (*tile, and the units before it as the result). No division per tile:
  // the token of a tile's last row advances by ROWS / group.
  __device__ static int64_t units_of(const AttnArgs& a, const KvSeq& s, int pad, int64_t want = -1, int* tile = nullptr) {
    const int nt = tiles_of(a, s), heads = a.c.kv_heads;
    if (nt == 1) {
      if (tile) *tile = 0;
      return want >= 0 ? 0 : (int64_t)span_of(max(1, (s.kv + UNIT - 1) / UNIT), pad) * heads;
    }
    const int g = a.c.group, dq = ROWS / g, dr = ROWS - dq * g;
    int q = (ROWS - 1) / g, r = ROWS - 1 - q * g;
    int64_t n = 0;
    for (int i = 0; i < nt; ++i) {
      const int see = a.causal && i + 1 < nt ? s.kv - s.n + q + 1 : s.kv;
      const int64_t u = (int64_t)span_of(max(1, (see + UNIT - 1) / UNIT), pad) * heads;
      if (want >= 0 && want < n + u) {
        *tile = i;
        return n;
      }
      n += u;
      q += dq;
      r += dr;
      if (r >= g) r -= g, ++q;
    }
    return n;
  }
  // Inclusive sum over the thread block (or, alone, the warp) of one value per
  // thread; *all its total.
  __device__ __forceinline__ static int64_t scan(int64_t x, int64_t* all, bool alone) {
    __shared__ int64_t wsum[WARPS];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int64_t y = __shfl_up_sync(0xffffffffu, x, o);
      if (lane >= o) x += y;
    }
    if (alone) {
      *all = __shfl_sync(0xffffffffu, x, 31);
      return x;
    }
    __syncthreads();  // an earlier call's readers are done
    if (lane == 31 && warp < WARPS) wsum[warp] = x;
    __syncthreads();
    int64_t t = 0;
#pragma unroll
    for (int w = 0; w < WARPS; ++w) {
      if (w < warp) x += wsum[w];
      t += wsum[w];
    }
    *all = t;
    return x;
  }
  // Finds the share of this thread block (every thread calls it); false when it
  // is empty. Where all (tile, head) pairs fit the launch in shares of min_units,
  // no share holds parts of two: short sequences are latency bound, and a share
  // across a boundary does two pairs' chains of loads one after the other. Up to
  // 32 sequences are one warp's work.
  __device__ bool start(const AttnArgs& a) {
    struct Found {
      KvSeq s;
      int b, pad;
      int64_t first, total;
    };
    __shared__ Found found;
    const KvArgs& c = a.c;
    constexpr int kN = 32 * WARPS;
    const bool alone = c.n_seq <= 32;
    if (!alone || threadIdx.x < 32) {
      KvSeq q{0, 0, 0};
      int64_t sum[2] = {0, 0}, all;  // units as they are, and padded
      for (int base = 0; base < c.n_seq; base += kN) {
        const int i = base + (int)threadIdx.x;
        q = KvSeq{0, 0, 0};
        if (threadIdx.x < kN && i < c.n_seq) q = kv_seq(c, i);
        if (q.n < 0 && blockIdx.x == 0) atomicOr(c.status, kFaultBatch);
        int64_t n = units_of(a, q, 1);
        scan(n, &all, alone);
        sum[0] += all;
        if (a.min_units > 1) {
          scan(units_of(a, q, a.min_units), &all, alone);
          sum[1] += all;
        }
      }
      pad = a.min_units > 1 && sum[1] <= (int64_t)a.min_units * gridDim.x ? a.min_units : 1;
      const int64_t total = sum[pad > 1];
      set_chunk(a, total);
      int64_t before = 0;
      for (int base = 0; base < c.n_seq; base += kN) {
        const int i = base + (int)threadIdx.x;
        if (c.n_seq > kN) q = threadIdx.x < kN && i < c.n_seq ? kv_seq(c, i) : KvSeq{0, 0, 0};
        const int64_t mine = units_of(a, q, pad), upto = before + scan(mine, &all, alone);
        before += all;
        if (u < upto && u >= upto - mine) found = Found{q, i, pad, upto - mine, total};
        if (u < before) break;
      }
      if (threadIdx.x == 0 && u >= total) found.total = total, found.pad = pad;
    }
    __syncthreads();
    pad = found.pad;
    set_chunk(a, found.total);
    if (u >= u_end) return false;
    b = found.b;
    s = found.s;
    tile_first = found.first + units_of(a, s, pad, u - found.first, &t);
    blocks = blocks_of(a, s, t);
    return true;
  }
  __device__ __forceinline__ void set_chunk(const AttnArgs& a, int64_t total) {
    const int64_t n = total + gridDim.x - 1;
    const int64_t even = n <= INT32_MAX ? (int)n / (int)gridDim.x : n / gridDim.x;
    chunk = pad > 1 ? pad : max((int64_t)a.min_units, even);
    u = chunk * blockIdx.x;
    u_end = min(total, u + chunk);
  }
  __device__ __forceinline__ bool more() const { return u < u_end; }
  __device__ __forceinline__ SegRec record(const Segment& g) const {
    return SegRec{b, g.h, g.blk0, g.blk1, t * ROWS, g.rows, s.first, s.n, s.kv, g.c0, g.c1, g.whole};
  }
  // The record of this segment, the walk moved past it. In a function of its own:
  // in line its registers cost the kernels theirs.
  __device__ __noinline__ static void next(UnitWalk* w, const AttnArgs& a, SegRec* rec) {
    rec->b = -1;
    while (w->more()) {
      const Segment g = w->segment(a);
      if (!g.empty) *rec = w->record(g);
      w->advance(a, g);
      if (!g.empty) return;
    }
  }
  __device__ __forceinline__ Segment segment(const AttnArgs& a) const {
    Segment g;
    const int span = span_of(blocks, pad);
    g.h = (int)(u - tile_first) / span;
    g.first = tile_first + (int64_t)g.h * span + lead();
    g.blk0 = max(0, (int)(u - g.first));
    g.blk1 = (int)min((int64_t)blocks, u_end - g.first);
    g.rows = min(ROWS, s.n * a.c.group - t * ROWS);
    g.empty = g.blk1 <= g.blk0;
    g.whole = g.blk0 == 0 && g.blk1 == blocks;
    // blocks before this share and from its end on, in shares (32-bit divisions)
    if (g.empty || g.whole) {
      g.c0 = g.c1 = blockIdx.x;
      return g;
    }
    const int share = (int)min(chunk, (int64_t)INT32_MAX);
    const int64_t u0 = chunk * blockIdx.x;
    g.c0 = g.first >= u0 ? (int)blockIdx.x : (int)blockIdx.x - ((int)(u0 - g.first) + share - 1) / share;
    const int64_t over = g.first + blocks - (u0 + chunk);
    g.c1 = over <= 0 ? (int)blockIdx.x : (int)blockIdx.x + ((int)over + share - 1) / share;
    return g;
  }
  __device__ __forceinline__ void advance(const AttnArgs& a, const Segment& g) {
    const int span = span_of(blocks, pad);
    u = g.blk1 >= blocks ? g.first - lead() + span : max(u + 1, g.first + g.blk1);
    if (u >= u_end || g.h + 1 < a.c.kv_heads) return;
    tile_first += (int64_t)span * a.c.kv_heads;
    if (++t >= tiles_of(a, s)) {
      t = 0;
      do {
        s = kv_seq(a.c, ++b);
      } while (s.n <= 0);  // units remain, so a sequence with rows follows
    }
    blocks = blocks_of(a, s, t);
  }
};

// Query rows row0 .. of a tile -> token and head within the group, without a
// division per row: x / group for x < group + 256 by multiplication, exact while
// x group < 2^22 (groups up to 1024; the entry point refuses larger ones).
struct RowMap {
  int tok0, rem0, group;
  uint32_t inv;
  __device__ __forceinline__ RowMap(const KvArgs& c, int row0) {
    group = c.group;
    tok0 = row0 / group;
    rem0 = row0 - tok0 * group;
    inv = (1u << 22) / (uint32_t)group + 1;
  }
  __device__ __forceinline__ void at(int i, int* tok, int* head) const {
    const int x = rem0 + i, q = (int)(((uint32_t)x * inv) >> 22);
    *tok = tok0 + q;
    *head = x - q * group;
  }
};

// The slot of thread block k's partial result of a tile that begins in c0's share.
__device__ __forceinline__ float* partial_slot(const AttnArgs& a, int k, int c0) {
  return a.partial + (int64_t)(2 * k + (k == c0 ? 1 : 0)) * a.slot_floats;
}

__device__ __forceinline__ float ex2(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

// A word whose first n bytes are ones.
__device__ __forceinline__ uint32_t first_bytes(int n) { return n >= 4 ? ~0u : (n <= 0 ? 0u : (1u << (8 * n)) - 1u); }

// Bulk copies bring blocks of tokens to shared memory, but for the keys of
// 16-token pages: pieces of 256 bytes took longer than the block's products (chunks
// that take 465 us from pages of 64 took 714 us, decode steps that take 66 us 77),
// so these go 16 bytes per lane.
__host__ __device__ __forceinline__ bool small_pages(const KvArgs& c) { return c.log_page == 4; }
__device__ __forceinline__ void copy16(void* dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(dst)), "l"(src) : "memory");
}
// Arrives at mb once this lane's copies so far are there.
__device__ __forceinline__ void copies_arrive(unsigned long long* mb) {
  asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"((uint32_t)__cvta_generic_to_shared(mb)) : "memory");
}
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_all;" ::: "memory"); }

// 4 codes -> binary16 pairs.
__device__ __forceinline__ void widen4(uint32_t w, uint32_t& lo, uint32_t& hi) {
  asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, l;\n\tcvt.rn.f16x2.e4m3x2 %1, h;\n\t}"
      : "=r"(lo), "=r"(hi)
      : "r"(w));
}

// 16 codes -> binary16 pairs in order.
__device__ __forceinline__ void widen(const uint4& v, uint32_t* f) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) widen4(w[i], f[2 * i], f[2 * i + 1]);
}

// These kernels' launches are set up while the kernel before them in the stream
// ends (append, attention and joining launch follow one another): every thread
// first waits for that kernel's end and its writes, so nothing is read early. 1 to 3
// us a call. What that kernel may write was not read-only for the whole life of this
// one, so it is read by ordinary loads, exponents past L1, never by non-coherent ones.
__device__ __forceinline__ void let_next_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void wait_for_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
template <typename K, typename A>
cudaError_t launch_next(K kernel, dim3 grid, int threads, size_t smem, const A& a, cudaStream_t st) {
  cudaLaunchAttribute attr{};
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, a);
}

// Row tiles a batch can have at most.
inline int64_t tiles_upper(const KvArgs& c, int tile_rows) {
  return (int64_t)c.n_tok * c.group / tile_rows + (c.n_seq < c.n_tok ? c.n_seq : c.n_tok);
}

cudaError_t launch_kv_append(const KvArgs& c, int head_dim, int dtype, const KvRows& q, const KvRows& k,
                             const KvRows& v, const KvRows& qo, const float* cos, const float* sin, int rope_rows,
                             int rotary_dim, int interleaved, cudaStream_t st);
cudaError_t launch_paged_rows(const AttnArgs& a, int head_dim, int dtype, int max_new, int max_kv, cudaStream_t st);
// A tile shared by several thread blocks, as the one it begins in leaves it for
// the joining kernel; rows = 0: none.
struct SharedTile {
  int row0, rows, first, h, c1, pad_[3];
};
cudaError_t launch_paged_tiles(const AttnArgs& a, int head_dim, int max_kv, cudaStream_t st);  // BF16

}  // namespace awsrc
