// step_plan.cu — the tables of a serving step from the requests' lengths: which
// pages come back and which are handed out, q_start, and each new token's
// sequence, position and slot.
//
// All sums are prefix sums over the sequences: needs and new tokens decide who
// finds room; pages given back, pages handed out and tokens got (of those who
// did) say where each page and token goes. Every thread block sums over all
// sequences (at most 8192) for itself; pages and tokens, numbered through, are dealt
// out over all threads, each finding its sequence by bisection of the sums in shared
// memory. Nobody waits for anybody: pages handed out that lie on the stack are not
// written by the call, those given back in it are taken from their old place in the
// table, which nobody writes. Only the lengths and the stack's count are read by
// all and written: by the thread block that was the last to have read them.
//
// Floor: some 16 bytes a token, far below the chain of loads and sums, 4 us of a small
// call. Measured: 8 sequences 4.9 us; 1000 sequences with 50 thousand tokens 8.3 us
// (one thread block 65, a cluster of 8 with barriers between its phases 13).
#include "internal.h"
#include "step.cuh"

namespace awsrc {

namespace {

// Sums of a block's threads before this one, and of all; three sums at a time.
struct Sum3 {
  int64_t a, b, c;
};
__device__ __forceinline__ int64_t warp_incl(int64_t v) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int64_t o = __shfl_up_sync(0xffffffffu, v, d);
    if (lane >= d) v += o;
  }
  return v;
}
template <int kThreads>
__device__ Sum3 block_excl(Sum3 v, Sum3* total, Sum3* warps) {
  constexpr int kWarps = kThreads / 32;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  __syncthreads();  // warps[] of the sum before is read
  const Sum3 i{warp_incl(v.a), warp_incl(v.b), warp_incl(v.c)};
  if (lane == 31) warps[warp] = i;
  __syncthreads();
  if (warp == 0) {
    const Sum3 w = lane < kWarps ? warps[lane] : Sum3{0, 0, 0};
    const Sum3 wi{warp_incl(w.a), warp_incl(w.b), warp_incl(w.c)};
    __syncwarp();
    if (lane < kWarps) warps[lane] = Sum3{wi.a - w.a, wi.b - w.b, wi.c - w.c};
    if (lane == 31) warps[32] = wi;
  }
  __syncthreads();
  *total = warps[32];
  const Sum3 before = warps[warp];
  return Sum3{before.a + i.a - v.a, before.b + i.b - v.b, before.c + i.c - v.c};
}

template <int kThreads>
struct Threads {};

struct Entry {
  int len, keep, add;  // add 0 and keep = len for an entry that cannot be right
  bool ok;
};

__device__ __forceinline__ int pages_of(int64_t tokens, int log_page) {
  return (int)((tokens + (1 << log_page) - 1) >> log_page);
}

__device__ __forceinline__ Entry load_entry(const PlanArgs& a, int b) {
  Entry e;
  e.len = a.len[b];
  e.keep = a.keep ? a.keep[b] : e.len;
  e.add = a.add[b];
  const int64_t most = (int64_t)a.stride << a.log_page;
  e.ok = e.len >= 0 && e.len <= most && e.keep >= 0 && e.keep <= e.len && e.add >= 0 && (int64_t)e.keep + e.add <= most;
  if (!e.ok) e.keep = e.len, e.add = 0;
  return e;
}

// Largest b with start[b] <= i, start[0] = 0: the sequence that item i belongs to
// (sequences without items are passed over).
__device__ __forceinline__ int find(const int* start, int n, int i) {
  int lo = 0, hi = n;  // start[lo] <= i < start[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (start[mid] <= i) lo = mid;
    else hi = mid;
  }
  return lo;
}

// Four maps' values from index t on.
template <typename T>
__device__ __forceinline__ void put4(T* p, int t, int n, bool vec, const T* v) {
  if (!p) return;
  if (vec && t + 4 <= n) {
    if (sizeof(T) == 4) {
      *reinterpret_cast<int4*>(p + t) = make_int4((int)v[0], (int)v[1], (int)v[2], (int)v[3]);
    } else {
      reinterpret_cast<longlong2*>(p + t)[0] = make_longlong2(v[0], v[1]);
      reinterpret_cast<longlong2*>(p + t)[1] = make_longlong2(v[2], v[3]);
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (t + i < n) p[t + i] = v[i];
}

// Needs and pages given back of a sequence, from shared memory.
__device__ __forceinline__ int want_of(int held, int keep, int add, int log_page) {
  return held < 0 ? 0 : pages_of((int64_t)keep + add, log_page);  // -1: an entry that cannot be right
}

// Page of the table's places [held, ..) that is handed out p-th.
struct Handed {
  const PlanArgs& a;
  const int *s_tok, *s_back, *s_keep;
  int count;
  __device__ __forceinline__ int operator()(int p) const {
    const int i = s_back[a.n_seq] - 1 - p;  // place above the old stack's top
    if (i < 0) return __ldcg(a.free + count + i);
    const int b = find(s_back, a.n_seq, i);
    return a.table[(int64_t)b * a.stride + pages_of((int64_t)s_keep[b] + s_tok[b + 1] - s_tok[b], a.log_page) + i - s_back[b]];
  }
};

template <int kThreads>
__global__ void __launch_bounds__(kThreads) plan_kernel(const __grid_constant__ PlanArgs a) {
  extern __shared__ int sm[];
  __shared__ Sum3 warps[33];
  __shared__ bool last;
  const int n = a.n_seq;
  int* s_tok = sm;               // n + 1: first token of a sequence (first: its new tokens)
  int* s_pop = sm + (n + 1);     // first page handed out
  int* s_back = sm + 2 * (n + 1);  // first page given back
  int* s_held = sm + 3 * (n + 1);  // pages held, -1 for an entry that cannot be right
  int* s_keep = sm + 4 * (n + 1);
  step_wait();
  step_trigger();
  const int tid = threadIdx.x, rank = blockIdx.x;
  const int count = *a.count;
  bool bad = false;
  for (int b = tid; b < n; b += kThreads) {
    const Entry e = load_entry(a, b);
    bad |= !e.ok;
    s_held[b] = e.ok ? pages_of(e.len, a.log_page) : -1;
    s_keep[b] = e.keep;
    s_tok[b] = e.add;
  }
  __syncthreads();
  if (tid == 0) {  // this block has read what the last one to say so writes
    unsigned said;
    asm volatile("atom.add.acq_rel.gpu.global.u32 %0, [%1], 1;" : "=r"(said) : "l"(a.arrived) : "memory");
    last = said == gridDim.x - 1;
    if (last) *a.arrived = 0;
  }
  const int per = (n + kThreads - 1) / kThreads;
  const int b0 = min(n, tid * per), b1 = min(n, b0 + per);
  Sum3 v{0, 0, 0}, total;
  for (int b = b0; b < b1; ++b) {
    const int held = max(0, s_held[b]), want = want_of(s_held[b], s_keep[b], s_tok[b], a.log_page);
    v.a += max(0, want - held);
    v.b += s_tok[b];
    v.c += max(0, held - want);
  }
  Sum3 before = block_excl<kThreads>(v, &total, warps);
  const int64_t room = count + total.c;
  bool short_ = false;
  if (total.a > room || total.b > a.n_tok) {  // not all find room: who does
    Sum3 got{0, 0, 0};
    for (int b = b0; b < b1; ++b) {
      const int held = max(0, s_held[b]), add = s_tok[b];
      int want = want_of(s_held[b], s_keep[b], add, a.log_page);
      before.a += max(0, want - held);
      before.b += add;
      if ((want > held && before.a > room) || before.b > a.n_tok) {
        short_ |= add > 0;
        s_tok[b] = 0;
        want = want_of(s_held[b], s_keep[b], 0, a.log_page);
      }
      got.a += max(0, want - held);
      got.b += s_tok[b];
      got.c += max(0, held - want);
    }
    before = block_excl<kThreads>(got, &total, warps);
  }
  const bool wrong = count < 0 || count > a.n_pages || count + total.c > a.n_pages;
  for (int b = b0; b < b1; ++b) {
    const int add = s_tok[b], held = max(0, s_held[b]), want = want_of(s_held[b], s_keep[b], add, a.log_page);
    s_pop[b] = (int)before.a;
    s_tok[b] = (int)before.b;
    s_back[b] = (int)before.c;
    before.a += max(0, want - held);
    before.b += add;
    before.c += max(0, held - want);
  }
  if (tid == 0) {
    s_pop[n] = (int)total.a;
    s_tok[n] = (int)total.b;
    s_back[n] = (int)total.c;
  }
  __syncthreads();
  const int step = gridDim.x * kThreads, at = rank * kThreads + tid;
  const uint32_t fault = (bad || wrong ? kFaultBatch : 0u) | (short_ ? kFaultRoom : 0u);
  if (rank == 0 && fault) atomicOr(a.status, fault);
  if (wrong) {
    for (int b = at; b <= n; b += step) a.q_start[b] = 0;
    for (int t = at; t < a.n_tok; t += step) {
      if (a.tok_seq) a.tok_seq[t] = -1;
      if (a.tok_pos) a.tok_pos[t] = -1;
      if (a.tok_slot) a.tok_slot[t] = -1;
    }
    return;
  }
  const int top = count + s_back[n];
  if (last) {
    for (int b = tid; b < n; b += kThreads) a.len[b] = s_keep[b] + s_tok[b + 1] - s_tok[b];
    if (tid == 0) *a.count = top - s_pop[n];
  }
  for (int b = at; b <= n; b += step) a.q_start[b] = s_tok[b];
  for (int i = at; i < s_back[n]; i += step) {
    const int b = find(s_back, n, i);
    const int want = pages_of((int64_t)s_keep[b] + s_tok[b + 1] - s_tok[b], a.log_page);
    a.free[count + i] = a.table[(int64_t)b * a.stride + want + i - s_back[b]];
  }
  const Handed handed{a, s_tok, s_back, s_keep, count};
  for (int i = at; i < s_pop[n]; i += step) {
    const int b = find(s_pop, n, i);
    a.table[(int64_t)b * a.stride + s_held[b] + i - s_pop[b]] = handed(i);
  }
  if (!a.tok_seq && !a.tok_pos && !a.tok_slot) return;
  // four tokens at a time: one bisection, mostly one page, and vector stores
  const int live = s_tok[n];
  for (int t0 = 4 * at; t0 < a.n_tok; t0 += 4 * step) {
    int seq[4], pos[4];
    int64_t slot[4];
    int b = t0 < live ? find(s_tok, n, t0) : n, page = 0, held_j = -1, held_b = -1;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int t = t0 + i;
      seq[i] = pos[i] = -1;
      slot[i] = -1;
      if (t >= live) continue;
      while (t >= s_tok[b + 1]) ++b;
      const int p = s_keep[b] + t - s_tok[b], j = p >> a.log_page;
      if (b != held_b || j != held_j) {
        held_b = b;
        held_j = j;
        page = j < s_held[b] ? a.table[(int64_t)b * a.stride + j] : handed(s_pop[b] + j - s_held[b]);
      }
      seq[i] = b;
      pos[i] = p;
      slot[i] = ((int64_t)page << a.log_page) + (p & (a.page - 1));
    }
    put4(a.tok_seq, t0, a.n_tok, a.vec, seq);
    put4(a.tok_pos, t0, a.n_tok, a.vec, pos);
    put4(a.tok_slot, t0, a.n_tok, a.vec, slot);
  }
}

template <int kThreads>
cudaError_t launch(const PlanArgs& a, cudaStream_t st) {
  const size_t smem = (size_t)5 * (a.n_seq + 1) * sizeof(int);
  if (smem > 46 * 1024) {
    const cudaError_t e = allow_smem<Threads<kThreads>>(plan_kernel<kThreads>, 5 * (kPlanMaxSeq + 1) * (int)sizeof(int));
    if (e != cudaSuccess) return e;
  }
  // a thread block for every four tokens of its threads, as many as SMs; each sums over all sequences
  const int64_t want = ((int64_t)a.n_tok + 4 * kThreads - 1) / (4 * kThreads);
  const int grid = (int)(want < 1 ? 1 : want > 152 ? 152 : want);
  return launch_step(plan_kernel<kThreads>, dim3(grid), kThreads, smem, 1, st, a);
}

}  // namespace

cudaError_t launch_plan(const PlanArgs& in, cudaStream_t st) {
  PlanArgs a = in;
  a.vec = ((reinterpret_cast<uintptr_t>(a.tok_seq) | reinterpret_cast<uintptr_t>(a.tok_pos) |
            reinterpret_cast<uintptr_t>(a.tok_slot)) & 15) == 0;
  // 8 sequences or more a thread in the sums are what a larger block is for; below, 8 warps: a
  // shuffle passes one warp per cycle, and 32 warps' sums took 4 us
  const cudaError_t e = a.n_seq <= 2048 ? launch<256>(a, st) : launch<1024>(a, st);
  if (e != cudaSuccess) return e;
  note_launches(1);
  return cudaGetLastError();
}

}  // namespace awsrc
