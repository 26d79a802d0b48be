// kv_append.cu — new keys and values into the paged 8-bit cache, q and k rotated
// by position on the way.
//
// Mathematics: a 2 x 2 rotation per pair, the block's amax -> one power-of-two
// exponent, e4m3 rounding. Per token it has to read (n_heads + 2 kv_heads) D
// elements and 2 (rotary_dim / 2) floats of the tables, and to write n_heads D
// elements and 2 kv_heads D codes: bytes bound, most of them q's. One launch
// does both parts, thread blocks of either kind alternating so that the waits of
// one pass under the other's bytes: a job is the keys or the values of one kv head
// and one page that gets tokens, by a warp where those are few or small pages,
// else by four; q is rotated by a few warps per token. A block's codes depend on
// its amax, so a job reads its tokens twice when they do not fit one item per
// thread (the second read hits L1/L2). Loads stand outside branches: behind one,
// each waited for the one before. Pages are found by a block-wide scan over the
// sequences, so the launch follows device-side lengths.
//
// Measured: 13k new tokens of 40 query and 8 kv heads (bf16, pages of 16) in 69 us,
// 4.9 TB/s of what it has to move; 8k tokens of 28 and 4 heads (pages of 64) in 33
// us, 4.7 TB/s. What is left is latency: a warp's loads (lengths, page, tables,
// rows) follow from one another, and rows that travel through registers leave 32
// warps an SM, at 64 of them. One token: 3.1 us a call in a captured run of them (6.2
// by itself).
//
// Rounding: the rotation in binary32, every operation rounded; q and k to q's type
// and to e4m3 once, codes in a scale that never lets them pass 448.
#include "internal.h"
#include "kv_paged.cuh"

namespace awsrc {

namespace {

constexpr int kThreads = 128;
constexpr int kWarps = kThreads / 32;

struct AppendArgs {
  KvArgs c;
  KvRows q, k, v, qo;
  const float *cos, *sin;
  int rope_rows, half, interleaved;  // half = rotary_dim / 2
  int kv_blocks, q_blocks, every;    // one block in `every` is of the kind with fewer
  int warps_per_tok;
};

// W consecutive elements.
template <int W>
__device__ __forceinline__ void load_row(const float* p, float* x) {
  if constexpr (W == 1) {
    x[0] = *p;
  } else {
#pragma unroll
    for (int i = 0; i < W; i += 4) {
      const float4 v = *reinterpret_cast<const float4*>(p + i);
      x[i] = v.x, x[i + 1] = v.y, x[i + 2] = v.z, x[i + 3] = v.w;
    }
  }
}
template <int W>
__device__ __forceinline__ void load_row(const __nv_bfloat16* p, float* x) {
  if constexpr (W == 1) {
    x[0] = __bfloat162float(*p);
  } else {
    static_assert(W == 8, "one 16-byte load");
    const uint4 v = *reinterpret_cast<const uint4*>(p);
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
  }
}
template <int W>
__device__ __forceinline__ void store_row(float* p, const float* x) {
  if constexpr (W == 1) {
    *p = x[0];
  } else {
#pragma unroll
    for (int i = 0; i < W; i += 4)
      *reinterpret_cast<float4*>(p + i) = make_float4(x[i], x[i + 1], x[i + 2], x[i + 3]);
  }
}
template <int W>
__device__ __forceinline__ void store_row(__nv_bfloat16* p, const float* x) {
  if constexpr (W == 1) {
    *p = __float2bfloat16_rn(x[0]);
  } else {
    uint4 v;
    uint32_t* w = &v.x;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    *reinterpret_cast<uint4*>(p) = v;
  }
}

// Element i of 8 in 16-byte vectors.
template <typename T>
__device__ __forceinline__ float element(const uint4* v, int i) {
  const uint32_t w[8] = {v[0].x, v[0].y, v[0].z, v[0].w, v[sizeof(T) / 4].x, v[sizeof(T) / 4].y, v[sizeof(T) / 4].z, v[sizeof(T) / 4].w};
  if constexpr (sizeof(T) == 2)
    return __uint_as_float(i & 1 ? w[i >> 1] & 0xFFFF0000u : w[i >> 1] << 16);
  else
    return __uint_as_float(w[i]);
}
template <typename T>
__device__ __forceinline__ void unpack(const uint4* v, float* x) {
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = element<T>(v, i);
}

// One item of a rotated head: W dims at d1 and, when `two`, their partners at d2.
template <int W>
struct Item {
  float y[2 * W];
  int d1, d2;
  bool two;
};

template <int W, int D>
__device__ __forceinline__ int items_per_head(const AppendArgs& a) {
  if (W == 8 && a.interleaved) return D / 8;
  return (D - a.half) / W;  // half / W pairs, then (D - 2 half) / W plain
}

__device__ __forceinline__ void turn(float& x1, float& x2, float c, float s) {
  const float a = __fsub_rn(__fmul_rn(x1, c), __fmul_rn(x2, s));
  x2 = __fadd_rn(__fmul_rn(x2, c), __fmul_rn(x1, s));
  x1 = a;
}

// Loads item `it` of the head at p and rotates it by the table rows cr, sr.
template <int W, typename T>
__device__ __forceinline__ void load_item(const AppendArgs& a, const T* p, int it, const float* cr, const float* sr,
                                          Item<W>& o) {
  const int h = a.half;
  const bool runs = W == 8 && a.interleaved;  // 4 pairs in 8 dims
  const bool turned = runs ? 8 * it < 2 * h : it * W < h;
  o.two = turned && !runs;
  o.d1 = runs ? 8 * it : (turned ? (a.interleaved ? 2 * it : it * W) : h + it * W);  // plain items: dims 2h on
  o.d2 = o.two ? (a.interleaved ? 2 * it + 1 : h + it * W) : o.d1;
  load_row<W>(p + o.d1, o.y);
  if (h == 0) return;
  float c[W], s[W];
  load_row<W>(p + o.d2, o.y + W);
  if (runs) {
    const int at = turned ? 4 * it : 0;
    load_row<4>(cr + at, c);
    load_row<4>(sr + at, s);
#pragma unroll
    for (int i = 0; i < W / 2; ++i) {
      float x1 = o.y[2 * i], x2 = o.y[2 * i + 1];
      turn(x1, x2, c[i], s[i]);
      o.y[2 * i] = turned ? x1 : o.y[2 * i];
      o.y[2 * i + 1] = turned ? x2 : o.y[2 * i + 1];
    }
  } else {
    const int at = turned ? it * W : 0;
    load_row<W>(cr + at, c);
    load_row<W>(sr + at, s);
#pragma unroll
    for (int i = 0; i < W; ++i) {
      float x1 = o.y[i];
      turn(x1, o.y[W + i], c[i], s[i]);
      o.y[i] = turned ? x1 : o.y[i];
    }
  }
}

template <int W>
__device__ __forceinline__ float item_amax(const Item<W>& o, float m) {
#pragma unroll
  for (int i = 0; i < W; ++i) m = fmax_nan(m, fabsf(o.y[i]));
  if (o.two) {
#pragma unroll
    for (int i = 0; i < W; ++i) m = fmax_nan(m, fabsf(o.y[W + i]));
  }
  return m;
}

// W key codes of dims d .. d + W - 1 of row `row`.
template <int W>
__device__ __forceinline__ void put_key(uint8_t* blk, int log_page, int row, int d, const float* y, float inv) {
  uint8_t* p = blk + ((((d >> 4) << log_page) + row) << 4) + (d & 15);
  if constexpr (W == 1) {
    *p = (uint8_t)e4m3x2(__fmul_rn(y[0], inv), 0.0f);
  } else {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = e4m3x2(__fmul_rn(y[2 * i], inv), __fmul_rn(y[2 * i + 1], inv));
    *reinterpret_cast<uint2*>(p) = make_uint2(w[0] | (w[1] << 16), w[2] | (w[3] << 16));
  }
}

// The sequence and page of visit number `visit` (pages that get new tokens,
// counted over the sequences in order). False past the last one. Visit 0 looks at
// all sequences and reports the entries that cannot be right.
__device__ __forceinline__ bool find_visit(const KvArgs& a, int visit, int* seq, int* nth) {
  __shared__ int wsum[kWarps], found[2];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int before = 0;
  if (threadIdx.x == 0) found[0] = -1;
  for (int base = 0; base < a.n_seq; base += kThreads) {
    const int b = base + threadIdx.x;
    int v = 0;
    if (b < a.n_seq) {
      const KvSeq s = kv_seq(a, b);
      if (s.n > 0) v = ((s.kv - 1) >> a.log_page) - ((s.kv - s.n) >> a.log_page) + 1;
      if (s.n < 0 && visit == 0) atomicOr(a.status, kFaultBatch);
    }
    int x = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, x, o);
      if (lane >= o) x += y;
    }
    if (lane == 31) wsum[warp] = x;
    __syncthreads();
    int off = before, all = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      if (w < warp) off += wsum[w];
      all += wsum[w];
    }
    if (visit >= off + x - v && visit < off + x) {
      found[0] = b;
      found[1] = visit - (off + x - v);
    }
    __syncthreads();
    before += all;
    if (visit > 0 && visit < before) break;
  }
  *seq = found[0];
  *nth = found[1];
  return found[0] >= 0;
}

// Over the JW warps of a job.
template <int JW>
__device__ __forceinline__ float job_amax(float m) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = fmax_nan(m, __shfl_xor_sync(0xffffffffu, m, o));
  if constexpr (JW > 1) {
    static_assert(JW == kWarps, "one job per thread block");
    __shared__ float wmax[kWarps];
    if ((threadIdx.x & 31) == 0) wmax[threadIdx.x >> 5] = m;
    __syncthreads();
    m = wmax[0];
#pragma unroll
    for (int w = 1; w < kWarps; ++w) m = fmax_nan(m, wmax[w]);
  }
  return m;
}

// 16 older codes: those with index < n become code * f.
__device__ __forceinline__ void rescale16(uint4* p, int n, float f) {
  uint4 v = *p;
  uint32_t* w = &v.x;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int sh = (i & 1) * 16;
    const uint32_t two = (w[i >> 1] >> sh) & 0xFFFFu;
    const uint32_t h = e4m3x2_half2(two);
    const float2 x = __half22float2(*reinterpret_cast<const __half2*>(&h));
    uint32_t r = e4m3x2(__fmul_rn(x.x, f), __fmul_rn(x.y, f));
    if (2 * i + 1 >= n) r = (r & 0xFFu) | (two & 0xFF00u);
    if (2 * i >= n) r = two;
    w[i >> 1] = (w[i >> 1] & ~(0xFFFFu << sh)) | (r << sh);
  }
  *p = v;
}

// The keys or values of one page visit (sequence b's nth) and kv head.
template <typename T, int D, int W, int JW>
__device__ void append_job(const AppendArgs& a, int b, int nth, int head, bool keys) {
  constexpr int kThreads = 32 * JW;  // of the job
  const KvArgs& c = a.c;
  const int tid = JW == 1 ? (int)(threadIdx.x & 31) : (int)threadIdx.x;
  const KvSeq s = kv_seq(c, b);
  const int P = 1 << c.log_page;
  const int first = s.kv - s.n;  // position of the first new token
  const int slot = (first >> c.log_page) + nth;
  const int pg = c.table[(int64_t)b * c.table_stride + slot];
  const int row0 = nth == 0 ? first & (P - 1) : 0;
  const int p0 = (slot << c.log_page) + row0;
  const int row1 = min(P, row0 + s.kv - p0);
  if (pg < 0 || pg >= c.n_pages || s.kv > a.rope_rows) {
    if (tid == 0) atomicOr(c.status, kFaultBatch);
    if (pg < 0 || pg >= c.n_pages) return;
  }
  // rows past the rotation tables are left out of keys and values alike
  const int n = min(row1 - row0, a.rope_rows - p0);
  if (n <= 0) return;
  const int tok0 = s.first + p0 - first;
  uint8_t* blk = (keys ? c.k : c.v) + block_off<D>(c, pg, head);
  int8_t* ep = (keys ? c.k_exp : c.v_exp) + (int64_t)pg * c.kv_heads + head;
  const int e_old = row0 ? (int)*ep : kExpMin;
  const int per = items_per_head<W, D>(a);
  // values: items of 4 rows x 8 dims (or single elements), so that codes leave in words
  const int g0 = row0 >> 2, groups = ((row0 + n - 1) >> 2) - g0 + 1;
  const int items = keys ? n * per : (W == 8 ? groups * (D / 8) : n * D);
  const KvRows& src = keys ? a.k : a.v;
  const T* sp = static_cast<const T*>(src.p) + (int64_t)head * src.hs;

  Item<W> it;
  constexpr int kV = sizeof(T) == 2 ? 1 : 2;  // 16-byte vectors of 8 elements
  uint4 vr[4][kV];                            // values: 4 rows as they came (in half the registers if bf16)
  float v1 = 0.0f;                            // or one element
  auto load = [&](int i) {
    if (keys) {
      const int t = i / per;
      const float* cr = a.cos + (int64_t)(p0 + t) * a.half;
      const float* sr = a.sin + (int64_t)(p0 + t) * a.half;
      load_item<W>(a, sp + (int64_t)(tok0 + t) * src.ts, i - t * per, cr, sr, it);
    } else if (W == 8) {
      const int r4 = (g0 + i / (D / 8)) * 4, d = i % (D / 8) * 8;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int r = r4 + j - row0;
        const uint4* p = reinterpret_cast<const uint4*>(  // a row of the job if not r
            sp + (int64_t)(tok0 + min(max(r, 0), n - 1)) * src.ts + d);
#pragma unroll
        for (int x = 0; x < kV; ++x) vr[j][x] = p[x];
      }
    } else {
      load_row<1>(sp + (int64_t)(tok0 + i / D) * src.ts + i % D, &v1);
    }
  };
  float m = 0.0f;
  for (int i = tid; i < items; i += kThreads) {
    load(i);
    if (keys) {
      m = item_amax<W>(it, m);
    } else if (W == 8) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        float y[8];
        unpack<T>(vr[j], y);
#pragma unroll
        for (int x = 0; x < 8; ++x) m = fmax_nan(m, fabsf(y[x]));
      }
    } else {
      m = fmax_nan(m, fabsf(v1));
    }
  }
  m = job_amax<JW>(m);
  const int need = block_exponent(m);
  const bool bad = need == kExpNan || e_old == kExpNan;
  const int e = bad ? kExpNan : max(need, e_old);
  if (tid == 0) *ep = (int8_t)e;
  if (!bad && row0 > 0 && e > e_old) {  // older codes in the new scale
    const float f = pow2f(e_old - e);
    uint4* q = reinterpret_cast<uint4*>(blk);
    if (keys) {
      for (int i = tid; i < (D / 16) * row0; i += kThreads)
        rescale16(q + ((i / row0) << c.log_page) + i % row0, 16, f);
    } else {
      for (int i = tid; i < ((row0 + 15) >> 4) * D; i += kThreads)
        rescale16(q + i, row0 - 16 * (i / D), f);
    }
    if constexpr (JW > 1)  // a 16-byte unit may get new codes too
      __syncthreads();
    else
      __syncwarp();
  }
  const float inv = bad ? 0.0f : pow2f(-e);
  for (int i = tid; i < items; i += kThreads) {
    if (items > kThreads) load(i);
    if (keys) {
      const int row = row0 + i / per;
      if (bad) {
#pragma unroll
        for (int x = 0; x < 2 * W; ++x) it.y[x] = 0.0f;
      }
      put_key<W>(blk, c.log_page, row, it.d1, it.y, inv);
      if (it.two) put_key<W>(blk, c.log_page, row, it.d2, it.y + W, inv);
    } else if (W == 8) {
      const int r4 = (g0 + i / (D / 8)) * 4, d = i % (D / 8) * 8;
      uint8_t* p = blk + ((int64_t)((r4 >> 4) * D + d) << 4) + (r4 & 15);
      const bool whole = r4 >= row0 && r4 + 4 <= row0 + n;
      if (bad) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int x = 0; x < kV; ++x) vr[j][x] = make_uint4(0, 0, 0, 0);
      }
#pragma unroll
      for (int x = 0; x < W; ++x) {
        const float y0 = element<T>(vr[0], x), y1 = element<T>(vr[1], x);
        const float y2 = element<T>(vr[2], x), y3 = element<T>(vr[3], x);
        const uint32_t w = e4m3x2(__fmul_rn(y0, inv), __fmul_rn(y1, inv)) |
                           (e4m3x2(__fmul_rn(y2, inv), __fmul_rn(y3, inv)) << 16);
        if (whole) {
          *reinterpret_cast<uint32_t*>(p + 16 * x) = w;
        } else {
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (r4 + j >= row0 && r4 + j < row0 + n) p[16 * x + j] = (uint8_t)(w >> (8 * j));
        }
      }
    } else {
      const int row = row0 + i / D, d = i % D;
      blk[(((row >> 4) * D + d) << 4) + (row & 15)] = (uint8_t)e4m3x2(__fmul_rn(bad ? 0.0f : v1, inv), 0.0f);
    }
  }
}

// Rotates part `part` of `parts` of token t's query heads (one warp).
template <typename T, int D, int W>
__device__ void rotate_q(const AppendArgs& a, int t, int part, int parts) {
  const KvArgs& c = a.c;
  const int lane = threadIdx.x & 31;
  // its sequence: the last one that starts at or before t
  int b = -1;
  for (int base = 0; base < c.n_seq; base += 32) {
    const bool le = base + lane < c.n_seq && c.q_start[base + lane] <= t;
    const unsigned m = __ballot_sync(0xffffffffu, le);
    if (m) b = base + 31 - __clz(m);
    if (m != 0xffffffffu) break;  // starts do not fall in a batch that can be right
  }
  KvSeq s{0, -1, 0};
  if (b >= 0) s = kv_seq(c, b);
  const int pos = s.kv - s.n + t - s.first;
  if (s.n < 0 || t >= s.first + s.n || pos >= a.rope_rows) {
    if (lane == 0) atomicOr(c.status, kFaultBatch);
    return;
  }
  const int per = items_per_head<W, D>(a);
  const float* cr = a.cos + (int64_t)pos * a.half;
  const float* sr = a.sin + (int64_t)pos * a.half;
  const T* qp = static_cast<const T*>(a.q.p) + (int64_t)t * a.q.ts;
  T* op = static_cast<T*>(a.qo.p) + (int64_t)t * a.qo.ts;
  if (W == 8 && !a.interleaved && a.half == D / 2) {
    // whole heads: a lane keeps its 8 pairs of the tables; kU heads in flight,
    // unpacked only when they are turned
    constexpr int kPer = D / 16, kHeads = 32 / kPer, kU = 2;  // lanes of a head, heads at a time
    constexpr int kV = sizeof(T) == 2 ? 1 : 2;                // 16-byte vectors of 8 elements
    const int it = lane % kPer;
    float cs[W], sn[W];
    load_row<W>(cr + W * it, cs);
    load_row<W>(sr + W * it, sn);
    const int step = parts * kHeads;
    for (int h0 = part * kHeads + lane / kPer; h0 < c.n_heads; h0 += kU * step) {
      uint4 raw[kU][2][kV];
#pragma unroll
      for (int u = 0; u < kU; ++u) {
        const uint4* p = reinterpret_cast<const uint4*>(qp + (int64_t)min(h0 + u * step, c.n_heads - 1) * a.q.hs + W * it);
#pragma unroll
        for (int j = 0; j < kV; ++j) raw[u][0][j] = p[j], raw[u][1][j] = p[D / 16 * kV + j];
      }
#pragma unroll
      for (int u = 0; u < kU; ++u) {
        float x[2 * W];
        unpack<T>(raw[u][0], x);
        unpack<T>(raw[u][1], x + W);
#pragma unroll
        for (int i = 0; i < W; ++i) turn(x[i], x[W + i], cs[i], sn[i]);
        if (h0 + u * step < c.n_heads) {
          T* o = op + (int64_t)(h0 + u * step) * a.qo.hs + W * it;
          store_row<W>(o, x);
          store_row<W>(o + D / 2, x + W);
        }
      }
    }
    return;
  }
  const int items = c.n_heads * per;
#pragma unroll 2
  for (int i = part * 32 + lane; i < items; i += parts * 32) {
    const int h = i / per;
    Item<W> it;
    load_item<W>(a, qp + (int64_t)h * a.q.hs, i - h * per, cr, sr, it);
    T* o = op + (int64_t)h * a.qo.hs;
    store_row<W>(o + it.d1, it.y);
    if (it.two) store_row<W>(o + it.d2, it.y + W);
  }
}

// Bytes in flight come from warps, not from deeper loops: at 13k tokens of 40
// heads (bf16) 3 thread blocks per SM with four heads in flight took 81 us, 6
// with two 76, 8 (64 registers) 72; unrolling the jobs' loops cost 10 us.
template <typename T, int D, int W, int JW>
__global__ void __launch_bounds__(kThreads, sizeof(T) == 2 ? 8 : 5) kv_append_kernel(const __grid_constant__ AppendArgs a) {
  wait_for_previous();
  let_next_start();
  // which kind, and the how many-th of it
  const int i = blockIdx.x, few = min(a.kv_blocks, a.q_blocks);
  const int nth = i / a.every, before = min(few, nth + (i % a.every != 0));  // blocks of the rarer kind up to i
  const bool rare = i % a.every == 0 && nth < few;
  const bool kv = rare == (a.kv_blocks <= a.q_blocks);
  const int k = rare ? nth : i - before;
  if (kv) {
    constexpr int kJobs = kWarps / JW;  // jobs of a thread block: of one visit
    const int jobs = 2 * a.c.kv_heads, per = (jobs + kJobs - 1) / kJobs;
    int b, visit;
    if (!find_visit(a.c, k / per, &b, &visit)) return;
    const int job = k % per * kJobs + (JW == 1 ? (int)(threadIdx.x >> 5) : 0);
    if (job < jobs) append_job<T, D, W, JW>(a, b, visit, job >> 1, (job & 1) == 0);
    return;
  }
  const int w = k * kWarps + (threadIdx.x >> 5);
  const int t = w / a.warps_per_tok;
  if (t < a.c.n_tok) rotate_q<T, D, W>(a, t, w % a.warps_per_tok, a.warps_per_tok);
}

template <typename T, int D>
cudaError_t launch(AppendArgs a, bool vec, int64_t visits, cudaStream_t st) {
  // A warp per job where a visit has few tokens (mean of the batch) or a small
  // page: 20 us less than four warps per job for 16k tokens in pages of 16.
  const bool warp = a.c.page <= 32 || (int64_t)a.c.n_tok <= 8 * visits;
  const int64_t jobs = 2ll * a.c.kv_heads, kv = visits * (warp ? (jobs + kWarps - 1) / kWarps : jobs);
  const int64_t q = ((int64_t)a.c.n_tok * a.warps_per_tok + kWarps - 1) / kWarps;
  if (kv + q > INT32_MAX) return cudaErrorInvalidValue;
  a.kv_blocks = (int)kv;
  a.q_blocks = (int)q;
  a.every = (int)((kv + q) / (kv < q ? kv : q));
  const unsigned grid = (unsigned)(kv + q);
  const auto kernel = vec ? (warp ? kv_append_kernel<T, D, 8, 1> : kv_append_kernel<T, D, 8, 4>)
                          : (warp ? kv_append_kernel<T, D, 1, 1> : kv_append_kernel<T, D, 1, 4>);
  note_launches(1);
  return launch_next(kernel, dim3(grid), kThreads, 0, a, st);
}

}  // namespace

cudaError_t launch_kv_append(const KvArgs& c, int head_dim, int dtype, const KvRows& q, const KvRows& k,
                             const KvRows& v, const KvRows& qo, const float* cos, const float* sin, int rope_rows,
                             int rotary_dim, int interleaved, cudaStream_t st) {
  AppendArgs a{};
  a.c = c;
  a.q = q;
  a.k = k;
  a.v = v;
  a.qo = qo;
  a.cos = cos;
  a.sin = sin;
  a.rope_rows = rotary_dim ? rope_rows : INT32_MAX;
  a.half = rotary_dim / 2;
  a.interleaved = interleaved;
  // pages that get tokens: a sequence of n tokens reaches at most n / page + 2
  // and at most n of them
  int64_t visits = (int64_t)c.n_tok / c.page + 2ll * c.n_seq;
  if (visits > c.n_tok) visits = c.n_tok;
  // a token's heads are shared by 4 warps while there are too few tokens for
  // one warp each to fill the GPU (152 SMs x 16 warps)
  a.warps_per_tok = c.n_tok >= 2432 ? 1 : kWarps;
  // vectors of 8 elements: every row, the tables and the rotated part in whole units
  const size_t elt = dtype == AWSRC_DTYPE_BF16 ? 2 : 4;
  const bool vec = rows_aligned(q, elt) && rows_aligned(k, elt) && rows_aligned(v, elt) && rows_aligned(qo, elt) &&
                   (reinterpret_cast<uintptr_t>(cos) | reinterpret_cast<uintptr_t>(sin)) % 16 == 0 &&
                   a.half % (interleaved ? 4 : 8) == 0;
  if (dtype == AWSRC_DTYPE_BF16)
    return head_dim == 128 ? launch<__nv_bfloat16, 128>(a, vec, visits, st) : launch<__nv_bfloat16, 64>(a, vec, visits, st);
  return head_dim == 128 ? launch<float, 128>(a, vec, visits, st) : launch<float, 64>(a, vec, visits, st);
}

}  // namespace awsrc
