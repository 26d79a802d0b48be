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

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kMaxCluster = 8;
typedef unsigned __int128 u128;

// A probability in units of 2^-62, rounded down; NaN and negative values 0, above 1 as 1.
__device__ __forceinline__ uint64_t units(float p) {
  const uint32_t u = __float_as_uint(fminf(fmaxf(p, 0.0f), 1.0f));  // NaN: 0
  const int e = (int)(u >> 23);
  const uint64_t m = (u & 0x7FFFFFu) | 0x800000u;
  return e >= 88 ? m << (e - 88) : e > 64 ? m >> (88 - e) : 0;
}

__device__ __forceinline__ float prob(const void* p, int64_t i, bool bf16) {
  return bf16 ? __bfloat162float(static_cast<const __nv_bfloat16*>(p)[i]) : static_cast<const float*>(p)[i];
}

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

struct Row {
  const void *p, *q;  // row of the target; of the draft, or null
  bool pb, qb;        // bf16
  int drop;           // column whose weight is 0 (a draft of certainty that was not accepted), or -1
  __device__ __forceinline__ uint64_t weight(int64_t j) const {
    const uint64_t w = units(prob(p, j, pb));
    if (j == drop) return 0;
    if (!q) return w;
    const uint64_t o = units(prob(q, j, qb));
    return w > o ? w - o : 0;
  }
};

__global__ void __launch_bounds__(kThreads) verify_kernel(const __grid_constant__ VerifyArgs a, int p_bf16, int q_bf16) {
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
          const float p = prob(a.p, t * a.ps + x, p_bf16), q = a.q ? prob(a.q, t * a.qs + x, q_bf16) : 1.0f, u = a.u[t];
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
  const size_t pe = p_bf16 ? 2 : 4, qe = q_bf16 ? 2 : 4;
  Row row{static_cast<const char*>(a.p) + t * a.ps * (int64_t)pe, nullptr, p_bf16 != 0, q_bf16 != 0, -1};
  if (stop < drafts) {
    if (a.q) row.q = static_cast<const char*>(a.q) + t * a.qs * (int64_t)qe;
    else row.drop = a.ids[t + 1];
  }
  // the run of a warp: whole 32s
  const int runs = size * kWarps;
  const int64_t run = ((int64_t)a.vocab + 32ll * runs - 1) / (32ll * runs) * 32;
  const int64_t j0 = min((int64_t)a.vocab, (rank * kWarps + warp) * run), j1 = min((int64_t)a.vocab, j0 + run);
  u128 total = 0, below = 0, mine = 0;
  for (int choice = 0; choice < 2; ++choice) {
    u128 sum = 0;
    for (int64_t j = j0 + lane; j < j1; j += 32) sum += row.weight(j);
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
    for (int64_t i0 = j0; i0 < j1; i0 += 32) {
      const int64_t j = i0 + lane;
      const u128 upto = sum + warp_incl(j < j1 ? (u128)row.weight(j) : (u128)0);
      const uint32_t hit = __ballot_sync(0xffffffffu, upto > at);
      if (hit) {
        if (lane == 0) tokens[stop] = (int)(i0 + __ffs(hit) - 1);
        break;
      }
      sum = shfl(upto, 31);
    }
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

}  // namespace

cudaError_t launch_verify(const VerifyArgs& a, int p_dtype, int q_dtype, cudaStream_t st) {
  const int size = kMaxCluster;
  const cudaError_t e = launch_step(verify_kernel, dim3((unsigned)(a.n_seq * size)), kThreads, 0, size, st, a,
                                    (int)(p_dtype == AWSRC_DTYPE_BF16), (int)(q_dtype == AWSRC_DTYPE_BF16));
  if (e != cudaSuccess) return e;
  note_launches(1);
  return cudaGetLastError();
}

}  // namespace awsrc
