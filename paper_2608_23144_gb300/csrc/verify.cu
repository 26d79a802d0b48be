// verify.cu — drafted tokens accepted or not against the target's probabilities,
// and the token that follows them, drawn by inverting the sums of its weights.
//
// Mathematics: draft x of a sequence is accepted when u q(x) < p(x) (compared
// exactly in binary64: a product of two binary32 values). At the first that is
// not, the token has the weights max(0, p - q); after the last, p. It is the
// smallest j with C_j > r C_V, C the running sum. Sums are of whole numbers
// (probabilities in units of 2^-45, rounded to nearest), so that they are exact in
// any order and the token does not depend on how the row is cut up. Given up for that:
// p and q are rounded before they are subtracted, by 2^-46 of probability an entry at
// most (4e-9 over a row of 2^18), and entries below are never drawn. Units of 2^-62 cost
// 64-bit shifts, 43 us where these take 17.
//
// Floor: one row of p and one of q per sequence (only the row that decides is
// read) at the copy rate; a small call is a chain of four loads (rows, ids,
// probabilities, the row) and the two passes below.
//
// At most 2^18 columns: the running sums have 63 bits, the table of the warps' steps
// (s_step) one entry per 512 columns.
//
// A cluster per sequence: its thread blocks sum equal slices of the row, each
// warp a run of it in steps of 512, exchange the slices' sums, and the warp in whose
// run the threshold falls reads the step again that it falls in. Units come out of
// two binary32 additions whose sums' bits count them (Units); 64-bit shifts of the
// significands took four times the instructions (43 us in place of 24).
//
// Measured: 64 sequences of up to 5 drafts over 151936 float32 probabilities 17.0 us
// (floor 8.6: 2 us of chain, 9 of rows on SMs with three or four blocks each, 5 of
// exchange, search and end), 15.5 where a model's are bf16; one of 151936 8.7 us, of 32000
// 4.8; 24 of 50257 in bf16 6.0 us. 64 of 50257 float32 9.8 us, and 11.5 where rows lie off
// 16 bytes, so that all loads are of one element.
#include "internal.h"
#include "step.cuh"

namespace awsrc {

namespace {

constexpr int kMaxThreads = 1024, kMaxWarps = kMaxThreads / 32;
constexpr int kMaxCluster = 8, kMaxVocab = 1 << 18;
constexpr int kGroup = 4;              // elements of a lane at a time, one vector load where rows allow it
constexpr int kPiece = 32 * kGroup;    // of a warp
constexpr int kAhead = 4;              // pieces whose loads are in flight together
constexpr int kStep = kAhead * kPiece;

// A probability p in [0, 1] in units of 2^-45, rounded to nearest even, as hi 2^23 + lo
// and a constant. p + 2 rounds p to units of 2^-22, which the sum's bits count; what is
// left, at most 2^-23 and exact, plus 3 2^-23 rounds to units of 2^-45 the same way.
struct Units {
  int hi, lo;
};
__device__ __forceinline__ Units units(float p) {
  const float t = __fadd_rn(p, 2.0f), rest = __fsub_rn(p, __fsub_rn(t, 2.0f));
  return Units{__float_as_int(t), __float_as_int(__fadd_rn(rest, 0x3p-23f))};
}
__device__ __forceinline__ float clean(float p) { return __saturatef(p); }  // to [0, 1], NaN: 0

__device__ __forceinline__ float value(float x) { return x; }
__device__ __forceinline__ float value(__nv_bfloat16 x) { return __bfloat162float(x); }

__device__ __forceinline__ uint64_t warp_incl(uint64_t v) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const uint64_t o = __shfl_up_sync(0xffffffffu, v, d);
    if (lane >= d) v += o;
  }
  return v;
}

__device__ __forceinline__ uint64_t peer_sum(uint64_t* own, uint32_t rank) {
  uint32_t addr, peer;
  asm("{ .reg .u64 t; cvta.to.shared.u64 t, %1; cvt.u32.u64 %0, t; }" : "=r"(addr) : "l"(own));
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(peer) : "r"(addr), "r"(rank));
  uint64_t v;
  asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(peer) : "memory");
  return v;
}

// 4 elements from j on, as they lie in memory; 0 past `have`.
template <typename T>
struct Raw {
  uint32_t w[sizeof(T)];
};
template <bool kVec>
__device__ __forceinline__ Raw<float> group(const float* p, int j, int have) {
  Raw<float> r;
  if (kVec && have >= kGroup) {
    const uint4 v = __ldcg(reinterpret_cast<const uint4*>(p + j));
    r.w[0] = v.x, r.w[1] = v.y, r.w[2] = v.z, r.w[3] = v.w;
  } else {
#pragma unroll
    for (int i = 0; i < kGroup; ++i) r.w[i] = i < have ? __float_as_uint(p[j + i]) : 0u;
  }
  return r;
}
template <bool kVec>
__device__ __forceinline__ Raw<__nv_bfloat16> group(const __nv_bfloat16* p, int j, int have) {
  Raw<__nv_bfloat16> r;
  if (kVec && have >= kGroup) {
    const uint2 v = __ldcg(reinterpret_cast<const uint2*>(p + j));
    r.w[0] = v.x, r.w[1] = v.y;
  } else {
    const unsigned short* h = reinterpret_cast<const unsigned short*>(p + j);
#pragma unroll
    for (int i = 0; i < 2; ++i) r.w[i] = (2 * i < have ? h[2 * i] : 0u) | (2 * i + 1 < have ? (uint32_t)h[2 * i + 1] << 16 : 0u);
  }
  return r;
}
__device__ __forceinline__ float at(const Raw<float>& r, int i) { return clean(__uint_as_float(r.w[i])); }
__device__ __forceinline__ float at(const Raw<__nv_bfloat16>& r, int i) {
  return clean(__uint_as_float(i & 1 ? r.w[i >> 1] & 0xFFFF0000u : r.w[i >> 1] << 16));
}

// The row that decides: weights p less q (kDiff), or p but for at most one column.
template <typename P, typename Q>
struct Row {
  const P* p;
  const Q* q;     // row of the draft model
  int drop;       // column whose weight is 0 (a draft of certainty that was not accepted), or -1
};

// kAhead pieces of the row from j0 on, up to j1: f(piece, hi, lo) with the units of the
// lane's 4 weights; true ends the walk.
template <bool kVec, bool kDiff, typename P, typename Q, typename F>
__device__ __forceinline__ void pieces(const Row<P, Q>& r, int j0, int j1, F&& f) {
  const int lane = threadIdx.x & 31;
  Raw<P> p[kAhead];
  Raw<Q> q[kAhead];
#pragma unroll
  for (int i = 0; i < kAhead; ++i) {
    const int j = j0 + i * kPiece + lane * kGroup;
    p[i] = group<kVec>(r.p, j, j1 - j);
    if (kDiff) q[i] = group<kVec>(r.q, j, j1 - j);
  }
#pragma unroll
  for (int i = 0; i < kAhead; ++i) {
    int hi[kGroup], lo[kGroup];
#pragma unroll
    for (int k = 0; k < kGroup; ++k) {
      const float a = at(p[i], k), b = kDiff ? at(q[i], k) : 0.0f;
      const Units ua = units(a), ub = units(b);
      const bool more = kDiff ? a > b : j0 + i * kPiece + lane * kGroup + k != r.drop;
      hi[k] = more ? ua.hi - ub.hi : 0;
      lo[k] = more ? ua.lo - ub.lo : 0;
    }
    if (f(i, hi, lo)) return;
  }
}

// Sum of a warp's run [j0, j1); the sums of its steps in step[].
template <bool kVec, bool kDiff, typename P, typename Q>
__device__ __forceinline__ uint64_t run_sum(const Row<P, Q>& row, int j0, int j1, uint64_t* step) {
  uint64_t sum = 0;
  for (int j = j0; j < j1; j += kStep, ++step) {
    int hi = 0, lo = 0;  // of 16 elements: far from 2^31
    pieces<kVec, kDiff>(row, j, j1, [&](int, const int* h, const int* l) {
#pragma unroll
      for (int k = 0; k < kGroup; ++k) hi += h[k], lo += l[k];
      return false;
    });
    uint64_t all = (uint64_t)(((int64_t)hi << 23) + lo);
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) all += __shfl_xor_sync(0xffffffffu, all, d);
    if ((threadIdx.x & 31) == 0) *step = all;
    sum += all;
  }
  return sum;
}

// The first element of the step from j on whose running sum, `sum` before the step, is above bar; -1 on lanes that do not hold it.
template <bool kVec, bool kDiff, typename P, typename Q>
__device__ __forceinline__ int find_in(const Row<P, Q>& row, int j, int j1, uint64_t sum, uint64_t bar) {
  const int lane = threadIdx.x & 31;
  int found = -1;
  pieces<kVec, kDiff>(row, j, j1, [&](int i, const int* h, const int* l) {
    uint64_t w[kGroup], own = 0;
#pragma unroll
    for (int k = 0; k < kGroup; ++k) own += w[k] = (uint64_t)(((int64_t)h[k] << 23) + l[k]);
    const uint64_t upto = sum + warp_incl(own);
    const uint32_t hit = __ballot_sync(0xffffffffu, upto > bar);
    sum = __shfl_sync(0xffffffffu, upto, 31);
    if (!hit) return false;
    if (lane == __ffs(hit) - 1) {
      uint64_t c = upto - own;
      int k = 0;
      for (; k < kGroup - 1; ++k) {
        c += w[k];
        if (c > bar) break;
      }
      found = j + i * kPiece + lane * kGroup + k;
    }
    return true;
  });
  return found;
}

// floor(r total), exactly: r is a whole number of 24 bits by 2^-s, and their product has 88
// bits. (r cut off to units of 2^-64 missed whole numbers by less than 2^-18 below 2^-40.)
// From 1 on the last weight is drawn.
__device__ __forceinline__ uint64_t threshold(float r, uint64_t total) {
  if (r >= 1.0f) return total - 1;
  if (!(r > 0.0f)) return 0;
  const uint32_t u = __float_as_uint(r), e = u >> 23;
  const uint64_t m = (u & 0x7FFFFFu) | (e ? 1u << 23 : 0u), lo = m * total, hi = __umul64hi(m, total);
  const int s = 150 - (int)max(e, 1u);  // 24 to 149
  return s < 64 ? hi << (64 - s) | lo >> s : s < 128 ? hi >> (s - 64) : 0;
}

template <typename P, typename Q, bool kVec>
__global__ void __launch_bounds__(kMaxThreads, 1) verify_kernel(const __grid_constant__ VerifyArgs a) {
  const P* probs_p = static_cast<const P*>(a.p);
  const Q* probs_q = static_cast<const Q*>(a.q);
  __shared__ uint64_t s_warp[kMaxWarps];
  __shared__ uint64_t s_step[kMaxVocab / kStep];  // sums of the warps' steps
  __shared__ uint64_t s_all[2];  // this block's sum, of the first and of the second choice of weights
  __shared__ int s_stop;
  step_wait();
  step_trigger();
  const int size = (int)(gridDim.x / a.n_seq), b = blockIdx.x / size, rank = blockIdx.x % size;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
  const int first = a.row_start[b], end = a.row_start[b + 1];
  const int drafts = end - first - 1;
  int32_t* tokens = a.tokens + (int64_t)b * (a.max_draft + 1);
  if (first < 0 || end < first || end > a.n_rows || drafts > a.max_draft || drafts < 0) {  // the same for the whole cluster
    if (rank == 0) {
      for (int i = threadIdx.x; i <= a.max_draft; i += blockDim.x) tokens[i] = -1;
      if (threadIdx.x == 0) {
        a.accepted[b] = 0;
        if (a.keep) a.keep[b] = a.kv_len[b];
        if (!(first >= 0 && end == first && end <= a.n_rows)) atomicOr(a.status, kFaultBatch);
      }
    }
    return;
  }
  if (warp == 0) {
    int stop = drafts;
    // up to the first refused; the ids behind it are looked at all the same
    for (int i0 = 0; i0 < drafts && (stop == drafts || rank == 0); i0 += 32) {
      const int i = i0 + lane;
      const int64_t t = first + i;
      const int x = i < drafts ? a.ids[t + 1] : 0;
      const bool outside = x < 0 || x >= a.vocab;
      if (outside && rank == 0) atomicOr(a.status, kFaultBatch);
      if (stop < drafts) continue;
      bool refuse = outside;
      if (i < drafts && !outside) {
        const float p = value(probs_p[t * a.ps + x]), q = a.q ? value(probs_q[t * a.qs + x]) : 1.0f, u = a.u[t];
        refuse = !((double)fmaxf(u, 0.0f) * (double)clean(q) < (double)clean(p));
      }
      const uint32_t no = __ballot_sync(0xffffffffu, refuse);
      if (no) stop = i0 + __ffs(no) - 1;
    }
    if (lane == 0) s_stop = stop;
  }
  __syncthreads();
  const int stop = s_stop;
  const int64_t t = first + stop;
  Row<P, Q> row{probs_p + t * a.ps, nullptr, -1};
  if (stop < drafts) {
    if (a.q) row.q = probs_q + t * a.qs;
    else row.drop = a.ids[t + 1];
  }
  // the run of a warp: whole pieces
  const int runs = size * warps;
  const int run = (a.vocab + kPiece * runs - 1) / (kPiece * runs) * kPiece;
  const int j0 = min(a.vocab, (rank * warps + warp) * run), j1 = min(a.vocab, j0 + run);
  uint64_t total = 0, below = 0, mine = 0;
  uint64_t* step = s_step + warp * ((run + kStep - 1) / kStep);
  for (int choice = 0; choice < 2; ++choice) {
    mine = row.q ? run_sum<kVec, true>(row, j0, j1, step) : run_sum<kVec, false>(row, j0, j1, step);
    if (lane == 0) s_warp[warp] = mine;
    __syncthreads();
    if (threadIdx.x == 0) {
      uint64_t all = 0;
      for (int w = 0; w < warps; ++w) all += s_warp[w];
      s_all[choice] = all;
    }
    cluster_sync();
    total = below = 0;
    for (int c = 0; c < size; ++c) {
      const uint64_t part = peer_sum(&s_all[choice], c);
      if (c < rank) below += part;
      total += part;
    }
    if (total != 0 || (!row.q && row.drop < 0)) break;
    row.q = nullptr;
    row.drop = -1;
  }
  for (int w = 0; w < warp; ++w) below += s_warp[w];
  const uint64_t bar = threshold(a.r[b], total);
  if (total != 0 && below <= bar && bar < below + mine) {
    // the step that it falls in, and its elements again
    uint64_t sum = below;
    int j = j0;
    for (; sum + *step <= bar; j += kStep) sum += *step++;
    const int token = row.q ? find_in<kVec, true>(row, j, j1, sum, bar) : find_in<kVec, false>(row, j, j1, sum, bar);
    if (token >= 0) tokens[stop] = token;
  }
  if (rank == 0) {
    for (int i = threadIdx.x; i <= a.max_draft; i += blockDim.x)
      if (i != stop) tokens[i] = i < stop ? a.ids[first + 1 + i] : -1;
      else if (total == 0) tokens[i] = -1;
    if (threadIdx.x == 0) {
      a.accepted[b] = stop;
      if (a.keep) a.keep[b] = a.kv_len[b] - (drafts - stop);
    }
  }
  cluster_sync();  // no block leaves while others may read its sums
}

template <typename P, typename Q, bool kVec>
cudaError_t launch(const VerifyArgs& a, cudaStream_t st) {
  // all SMs for few sequences, up to 1024 threads each while a warp has a whole step;
  // 8 blocks a sequence while they run at the same time, four an SM (300 sequences of
  // 32000 elements: 2 blocks 13.3 us, 4: 19.6, 8: 27.6)
  int size = kMaxCluster, threads = kMaxThreads;
  while (threads > 256 && ((int64_t)a.n_seq * size * threads > 152 * 1024 || a.vocab < size * threads / 32 * kStep)) threads /= 2;
  while (size > 1 && (int64_t)a.n_seq * size > 4 * 152) size /= 2;
  return launch_step(verify_kernel<P, Q, kVec>, dim3((unsigned)(a.n_seq * size)), threads, 0, size, st, a);
}
template <typename P, typename Q>
cudaError_t launch(const VerifyArgs& a, cudaStream_t st) {
  // every group of 4 elements starts on a boundary of its size
  const bool vec = (reinterpret_cast<uintptr_t>(a.p) | (uintptr_t)(a.ps * (int64_t)sizeof(P))) % (kGroup * sizeof(P)) == 0 &&
                   (reinterpret_cast<uintptr_t>(a.q) | (uintptr_t)(a.qs * (int64_t)sizeof(Q))) % (kGroup * sizeof(Q)) == 0;
  return vec ? launch<P, Q, true>(a, st) : launch<P, Q, false>(a, st);
}

}  // namespace

cudaError_t launch_verify(const VerifyArgs& a, int p_dtype, int q_dtype, cudaStream_t st) {
  const bool pb = p_dtype == AWSRC_DTYPE_BF16, qb = a.q ? q_dtype == AWSRC_DTYPE_BF16 : pb;
  const cudaError_t e = pb ? (qb ? launch<__nv_bfloat16, __nv_bfloat16>(a, st) : launch<__nv_bfloat16, float>(a, st))
                           : (qb ? launch<float, __nv_bfloat16>(a, st) : launch<float, float>(a, st));
  if (e != cudaSuccess) return e;
  note_launches(1);
  return cudaGetLastError();
}

}  // namespace awsrc
