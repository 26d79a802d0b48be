// step.cuh — what the serving-step kernels (plan, verification, 8-bit products)
// share: their arguments and the launch that overlaps the kernel before.
#pragma once

#include <atomic>

#include "common.cuh"

namespace awsrc {

// Programmatic dependent launch, as the paged cache's kernels use it: a launch is
// set up while the kernel before it in the stream ends, and every thread waits
// for that kernel and its writes before it reads anything that may be written.
// Such memory is read by ordinary loads, never by non-coherent ones.
__device__ __forceinline__ void step_trigger() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void step_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

// A launch of clusters of `cluster` thread blocks along x.
template <typename K, typename... A>
cudaError_t launch_step(K kernel, dim3 grid, int threads, size_t smem, int cluster, cudaStream_t st, const A&... a) {
  cudaLaunchAttribute attr[2]{};
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = cluster;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cfg.attrs = attr;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kernel, a...);
}

// Lets a kernel use `bytes` of shared memory: once per device and kernel (K: a type of
// its own for each, such as its configuration).
template <typename K, typename F>
cudaError_t allow_smem(F kernel, int bytes) {
  static std::atomic<uint64_t> done{0};
  int dev = 0;
  const cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 64 && (done.load(std::memory_order_relaxed) >> dev & 1)) return cudaSuccess;
  const cudaError_t s = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (s == cudaSuccess && dev < 64) done.fetch_or(1ull << dev, std::memory_order_relaxed);
  return s;
}

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
// All threads of the cluster arrive; writes before are seen by reads after.
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// ---- plan (step_plan.cu)
constexpr int kPlanMaxSeq = 8192;
struct PlanArgs {
  int n_pages, page, log_page, n_seq, stride, n_tok;
  int32_t *table, *len, *free, *count;
  const int32_t *keep, *add;
  int32_t *q_start, *tok_seq, *tok_pos;
  int64_t* tok_slot;
  uint32_t* status;
  uint32_t* arrived;  // thread blocks that have read the lengths: 0 between calls
  int vec;            // the maps start on 16-byte boundaries
};
cudaError_t launch_plan(const PlanArgs& a, cudaStream_t st);

// ---- verification (verify.cu)
struct VerifyArgs {
  int n_seq, n_rows, vocab, max_draft;
  const int32_t *row_start, *ids;
  const void *p, *q;  // q null: drafts of certainty
  int64_t ps, qs;
  const float *u, *r;
  const int32_t* kv_len;
  int32_t *accepted, *tokens, *keep;
  uint32_t* status;
};
cudaError_t launch_verify(const VerifyArgs& a, int p_dtype, int q_dtype, cudaStream_t st);

// ---- 8-bit matrices and their product (fp8_quantize.cu, fp8_gemm.cu)
struct Fp8Mat {
  int rows, cols;
  uint8_t *codes, *exps;
  __host__ __device__ int blocks() const { return (cols + 127) >> 7; }
  __host__ __device__ int rows8() const { return (rows + 7) & ~7; }
  __host__ __device__ int tiles() const { return (rows + 127) >> 7; }
};
cudaError_t launch_fp8_quantize(const void* x, int dtype, int64_t stride, const Fp8Mat& m, cudaStream_t st);
struct GemmArgs {
  Fp8Mat x, w;
  void* y;
  int64_t ys;
  int y_f32;         // y is binary32, else bf16
  const void* raw;   // x before quantising, when the product does that itself (few rows); else null
  int64_t raw_stride;
  int raw_bf16;
  uint32_t* status;
  uint64_t wait_ns;  // limit of the kernel's waits
  int stall;         // test of that limit: no copies from this block of 128 columns on (-1: never)
  int early;         // w was written before the kernel before this one began: its rows need no wait
  // set by the launch
  int split;         // thread blocks (pairs of them) that share a tile's columns
  int n;             // rows of x in a tile; of w in the kernel for few rows of x
  int vec_y;         // four elements of y lie on a boundary of their size
  int vec_raw;       // so do four of every row of x
};
// Whether the product quantises these rows of x, float32 or bf16, itself (fp8_gemm.cu).
cudaError_t fp8_gemm_quantizes(const GemmArgs& a, bool bf16, bool* itself);
cudaError_t launch_fp8_pairs(const GemmArgs& a, cudaStream_t st);
cudaError_t launch_fp8_gemm(const GemmArgs& a, cudaStream_t st);

}  // namespace awsrc
