// verify.cu — drafted tokens accepted or not against the target's probabilities,
// and the token that follows them, drawn by inverting the sums of its weights.
//
// Mathematics: draft x of a sequence is accepted when u q(x) < p(x) (compared
// exactly in binary64: a product of two binary32 values). At the first that is
// not, the token has the weights max(0, p - q); after the last, p. It is the
// smallest j with C_j > r C_V, C the running sum. Sums are of whole numbers
// (probabilities in units of 2^-62, rounded down), so that they are exact in any
// order and the token does not depend on how the row is cut up.
//
// Floor: one row of p and one of q per sequence (only the row that decides is
// read) at the copy rate; a small call is a chain of four loads (rows, ids,
// probabilities, the row) and the two passes below.
//
// A cluster per sequence: its thread blocks sum equal slices of the row, each
// warp a run of it, exchange the slices' sums, and the warp in whose run the
// threshold falls reads that run again and finds the token.
#include "internal.h"
#include "step.cuh"

namespace awsrc {

namespace {

constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kMaxCluster = 8;
constexpr int kGroup = 4;              // elements of a lane at a time, one vector load where rows allow it
constexpr int kPiece = 32 * kGroup;    // of a warp
constexpr int kAhead = 4;              // pieces whose loads are in flight together
typedef unsigned __int128 u128;

// A probability in units of 2^-62, rounded down; NaN and negative values 0, above 1
// as 1. With the significand M in 32 bits and k = 128 - exponent, M 2^32 >> k; shifts
// by 32 or more, or by a negative amount, give 0 (PTX's clamp), so the low word needs
// no choice between its two forms.
__device__ __forceinline__ uint32_t shl(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("shl.b32 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ uint32_t shr(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("shr.u32 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ uint64_t units(float p) {
  const uint32_t u = __float_as_uint(fminf(fmaxf(p, 0.0f), 1.0f));  // NaN: 0
  const uint32_t m = (u << 8) | 0x80000000u, k = 128u - (u >> 23);
  const uint32_t hi = shr(m, k), lo = shl(m, 32u - k) | shr(m, k - 32u);
  return ((uint64_t)hi << 32) | lo;
}

__device__ __forceinline__ float value(float x) { return x; }
__device__ __forceinline__ float value(__nv_bfloat16 x) { return __bfloat162float(x); }

__device__ __forceinline__ u128 shfl(u128 v, int lane) {
  const uint64_t lo = __shfl_sync(0xffffffffu, (uint64_t)v, lane), hi = __shfl_sync(0xffffffffu, (uint64_t)(v >> 64), lane);
  return ((u128)hi << 64) | lo;
}
__device__ __forceinline__ u128 warp_incl(u128 v) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const uint64_t lo = __shfl_up_sync(0xffffffffu, (uint64_t)v, d), hi = __shfl_up_sync(0xffffffffu, (uint64_t)(v >> 64), d);
    if (lane >= d) v += ((u128)hi << 64) | lo;
  }
  return v;
}

__device__ __forceinline__ u128 peer_sum(u128* own, uint32_t rank) {
  uint32_t addr, peer;
  asm("{ .reg .u64 t; cvta.to.shared.u64 t, %1; cvt.u32.u64 %0, t; }" : "=r"(addr) : "l"(own));
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(peer) : "r"(addr), "r"(rank));
  uint64_t lo, hi;
  asm volatile("ld.shared::cluster.v2.u64 {%0, %1}, [%2];" : "=l"(lo), "=l"(hi) : "r"(peer) : "memory");
  return ((u128)hi << 64) | lo;
}

// 4 elements from j on; 0 past `have`.
template <bool kVec>
__device__ __forceinline__ float4 group(const float* p, int64_t j, int64_t have) {
  if (kVec && have >= kGroup) return __ldcg(reinterpret_cast<const float4*>(p + j));
  return make_float4(have > 0 ? p[j] : 0.0f, have > 1 ? p[j + 1] : 0.0f, have > 2 ? p[j + 2] : 0.0f, have > 3 ? p[j + 3] : 0.0f);
}
template <bool kVec>
__device__ __forceinline__ float4 group(const __nv_bfloat16* p, int64_t j, int64_t have) {
  if (kVec && have >= kGroup) {
    const uint2 x = __ldcg(reinterpret_cast<const uint2*>(p + j));
    return make_float4(__uint_as_float(x.x << 16), __uint_as_float(x.x & 0xFFFF0000u), __uint_as_float(x.y << 16),
                       __uint_as_float(x.y & 0xFFFF0000u));
  }
  return make_float4(have > 0 ? __bfloat162float(p[j]) : 0.0f, have > 1 ? __bfloat162float(p[j + 1]) : 0.0f,
                     have > 2 ? __bfloat162float(p[j + 2]) : 0.0f, have > 3 ? __bfloat162float(p[j + 3]) : 0.0f);
}

// The row that decides: weights p, p less q, or p but for one column.
template <typename P, typename Q>
struct Row {
  const P* p;
  const Q* q;     // row of the draft model, or null
  int64_t vocab;
  int64_t drop;   // column whose weight is 0 (a draft of certainty that was not accepted), or -1
};

__device__ __forceinline__ uint64_t weight(float p, float q) {
  const uint64_t w = units(p), o = units(q);
  return w > o ? w - o : 0;
}

// kAhead pieces of the row from j0 on, up to j1: each lane's weights.
template <bool kVec, typename P, typename Q, typename F>
__device__ __forceinline__ void pieces(const Row<P, Q>& r, int64_t j0, int64_t j1, F&& f) {
  const int lane = threadIdx.x & 31;
  float4 p[kAhead], q[kAhead];
#pragma unroll
  for (int i = 0; i < kAhead; ++i) {
    const int64_t j = j0 + i * kPiece + lane * kGroup;
    p[i] = group<kVec>(r.p, j, j1 - j);
    q[i] = r.q ? group<kVec>(r.q, j, j1 - j) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  }
#pragma unroll
  for (int i = 0; i < kAhead; ++i) {
    const int64_t at = r.drop - (j0 + i * kPiece + lane * kGroup);
    uint64_t w[kGroup] = {weight(p[i].x, q[i].x), weight(p[i].y, q[i].y), weight(p[i].z, q[i].z), weight(p[i].w, q[i].w)};
    if (at >= 0 && at < kGroup) {
#pragma unroll
      for (int k = 0; k < kGroup; ++k)
        if (k == at) w[k] = 0;
    }
    if (f(i, w)) return;
  }
}

template <typename P, typename Q, bool kVec>
__global__ void __launch_bounds__(kThreads, 2) verify_kernel(const __grid_constant__ VerifyArgs a) {
  const P* probs_p = static_cast<const P*>(a.p);
  const Q* probs_q = static_cast<const Q*>(a.q);
  __shared__ u128 s_warp[kWarps];
  __shared__ u128 s_all[2];  // this block's sum, of the first and of the second choice of weights
  __shared__ int s_stop;
  step_wait();
  step_trigger();
  const int size = (int)(gridDim.x / a.n_seq), b = blockIdx.x / size, rank = blockIdx.x % size;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int first = a.row_start[b], end = a.row_start[b + 1];
  const int drafts = end - first - 1;
  int32_t* tokens = a.tokens + (int64_t)b * (a.max_draft + 1);
  if (first < 0 || end < first || end > a.n_rows || drafts > a.max_draft || drafts < 0) {  // the same for the whole cluster
    if (rank == 0) {
      for (int i = threadIdx.x; i <= a.max_draft; i += kThreads) tokens[i] = -1;
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
    for (int i0 = 0; i0 < drafts && stop == drafts; i0 += 32) {
      const int i = i0 + lane;
      bool refuse = false;
      if (i < drafts) {
        const int64_t t = first + i;
        const int x = a.ids[t + 1];
        refuse = true;
        if (x >= 0 && x < a.vocab) {
          const float p = value(probs_p[t * a.ps + x]), q = a.q ? value(probs_q[t * a.qs + x]) : 1.0f, u = a.u[t];
          const float pc = fminf(fmaxf(p, 0.0f), 1.0f), qc = fminf(fmaxf(q, 0.0f), 1.0f), uc = fmaxf(u, 0.0f);
          refuse = !((double)uc * (double)qc < (double)pc);
        } else if (rank == 0) {
          atomicOr(a.status, kFaultBatch);
        }
      }
      const uint32_t no = __ballot_sync(0xffffffffu, refuse);
      if (no) stop = i0 + __ffs(no) - 1;
    }
    if (lane == 0) s_stop = stop;
  }
  __syncthreads();
  const int stop = s_stop;
  const int64_t t = first + stop;
  Row<P, Q> row{probs_p + t * a.ps, nullptr, a.vocab, -1};
  if (stop < drafts) {
    if (a.q) row.q = probs_q + t * a.qs;
    else row.drop = a.ids[t + 1];
  }
  // the run of a warp: whole pieces
  const int runs = size * kWarps;
  const int64_t run = ((int64_t)a.vocab + (int64_t)kPiece * runs - 1) / ((int64_t)kPiece * runs) * kPiece;
  const int64_t j0 = min((int64_t)a.vocab, (rank * kWarps + warp) * run), j1 = min((int64_t)a.vocab, j0 + run);
  u128 total = 0, below = 0, mine = 0;
  for (int choice = 0; choice < 2; ++choice) {
    u128 sum = 0;
    for (int64_t j = j0; j < j1; j += kAhead * kPiece)
      pieces<kVec>(row, j, j1, [&](int, const uint64_t* w) {
#pragma unroll
        for (int k = 0; k < kGroup; ++k) sum += w[k];
        return false;
      });
    mine = shfl(warp_incl(sum), 31);
    if (lane == 0) s_warp[warp] = mine;
    __syncthreads();
    if (threadIdx.x == 0) {
      u128 all = 0;
      for (int w = 0; w < kWarps; ++w) all += s_warp[w];
      s_all[choice] = all;
    }
    cluster_sync();
    total = below = 0;
    for (int c = 0; c < size; ++c) {
      const u128 part = peer_sum(&s_all[choice], c);
      if (c < rank) below += part;
      total += part;
    }
    if (total != 0 || (!row.q && row.drop < 0)) break;
    row.q = nullptr;
    row.drop = -1;
  }
  for (int w = 0; w < warp; ++w) below += s_warp[w];
  // floor(r total), r in units of 2^-64
  const float r = a.r[b];
  const uint64_t ru = r >= 1.0f ? ~0ull : r > 0.0f ? __float2ull_rz(__fmul_rn(r, 0x1p64f)) : 0;
  const u128 at = (u128)(uint64_t)(total >> 64) * ru + __umul64hi((uint64_t)total, ru);
  if (total != 0 && below <= at && at < below + mine) {
    u128 sum = below;
    bool found = false;
    for (int64_t j = j0; j < j1 && !found; j += kAhead * kPiece)
      pieces<kVec>(row, j, j1, [&](int i, const uint64_t* w) {
        u128 own = 0;
#pragma unroll
        for (int k = 0; k < kGroup; ++k) own += w[k];
        const u128 upto = sum + warp_incl(own);
        const uint32_t hit = __ballot_sync(0xffffffffu, upto > at);
        sum = shfl(upto, 31);
        if (!hit) return false;
        if (lane == __ffs(hit) - 1) {
          u128 c = upto - own;
          int k = 0;
          for (; k < kGroup - 1; ++k) {
            c += w[k];
            if (c > at) break;
          }
          tokens[stop] = (int)(j + i * kPiece + lane * kGroup + k);
        }
        return found = true;
      });
  }
  if (rank == 0) {
    for (int i = threadIdx.x; i <= a.max_draft; i += kThreads)
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
  return launch_step(verify_kernel<P, Q, kVec>, dim3((unsigned)(a.n_seq * kMaxCluster)), kThreads, 0, kMaxCluster, st, a);
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
