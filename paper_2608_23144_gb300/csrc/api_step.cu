// api_step.cu — the extern "C" entry points of serving steps declared in
// include/awsrc.h: argument validation and launches.
#include <climits>

#include "internal.h"
#include "step.cuh"

namespace awsrc {

namespace {

constexpr size_t kStepWorkspace = kStatusBytes;  // the fault word, and the plan's counter
constexpr int kArrivedAt = 32;

bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
bool is_dtype(int32_t d) { return d == AWSRC_DTYPE_F32 || d == AWSRC_DTYPE_BF16; }
uintptr_t size_of(int32_t dtype) { return dtype == AWSRC_DTYPE_BF16 ? 2 : 4; }

awsrc_status check_workspace(const void* ws, size_t bytes) {
  if (!ws || bytes < kStepWorkspace) return AWSRC_ERR_WORKSPACE;
  return aligned(ws, 256) ? AWSRC_OK : AWSRC_ERR_INVALID_ARG;
}

awsrc_status check_matrix(const awsrc_fp8_matrix* m, bool pointers, Fp8Mat* out) {
  if (!m || m->rows < 0) return AWSRC_ERR_INVALID_ARG;
  if (m->cols < 1) return AWSRC_ERR_SHAPE;
  if (m->rows > (1 << 30) || m->cols > (1 << 24)) return AWSRC_ERR_UNSUPPORTED;
  if (pointers && (!m->codes || !m->exps || !aligned(m->codes, 128) || !aligned(m->exps, 16))) return AWSRC_ERR_INVALID_ARG;
  *out = Fp8Mat{m->rows, m->cols, m->codes, m->exps};
  return AWSRC_OK;
}

awsrc_status check_rows(const void* x, int32_t dtype) {
  return is_dtype(dtype) && x && aligned(x, size_of(dtype)) ? AWSRC_OK : AWSRC_ERR_INVALID_ARG;
}

// Whether `rows` rows here and there share any byte. Rows at the same step may lie
// between each other's (columns of one wider matrix); at different steps their extents must not meet.
struct Rows {
  const void* p;
  int64_t step, row;  // bytes
};
bool share(const Rows& x, const Rows& y, int64_t rows) {
  const auto lo = [&](const Rows& m) { return (__int128)reinterpret_cast<uintptr_t>(m.p) + (m.step < 0 ? (rows - 1) * (__int128)m.step : 0); };
  const auto hi = [&](const Rows& m) { return (__int128)reinterpret_cast<uintptr_t>(m.p) + (m.step > 0 ? (rows - 1) * (__int128)m.step : 0) + m.row; };
  if (hi(x) <= lo(y) || hi(y) <= lo(x)) return false;
  if (rows == 1 || x.step != y.step || x.step == 0) return true;
  const __int128 step = x.step < 0 ? -(__int128)x.step : (__int128)x.step;
  __int128 d = ((__int128)reinterpret_cast<uintptr_t>(y.p) - (__int128)reinterpret_cast<uintptr_t>(x.p)) % step;
  if (d < 0) d += step;
  return d < x.row || step - d < y.row;
}

size_t codes_bytes(const Fp8Mat& m) { return (size_t)m.blocks() * m.rows8() * 128; }
size_t exps_bytes(const Fp8Mat& m) { return (size_t)((m.blocks() + 3) / 4) * m.tiles() * 512; }

// Whether two matrices held in 8 bits share a byte, of codes or of exponents.
bool share(const Fp8Mat& x, const Fp8Mat& w) {
  const auto meet = [](const uint8_t* a, size_t n, const uint8_t* b, size_t m) {
    const uintptr_t p = reinterpret_cast<uintptr_t>(a), q = reinterpret_cast<uintptr_t>(b);
    return n && m && (p <= q ? q - p < n : p - q < m);
  };
  return meet(x.codes, codes_bytes(x), w.codes, codes_bytes(w)) || meet(x.exps, exps_bytes(x), w.exps, exps_bytes(w)) ||
         meet(x.codes, codes_bytes(x), w.exps, exps_bytes(w)) || meet(x.exps, exps_bytes(x), w.codes, codes_bytes(w));
}

awsrc_status gemm_args(const awsrc_fp8_matrix* x, const awsrc_fp8_matrix* w, void* y, int32_t y_dtype, int64_t y_stride,
                       void* workspace, size_t workspace_bytes, GemmArgs* out) {
  GemmArgs a{};
  awsrc_status s;
  if ((s = check_matrix(x, true, &a.x)) != AWSRC_OK || (s = check_matrix(w, true, &a.w)) != AWSRC_OK ||
      (s = check_rows(y, y_dtype)) != AWSRC_OK)
    return s;
  if (x->cols != w->cols) return AWSRC_ERR_SHAPE;
  // rows of y that share elements would be written by several thread blocks
  if (x->rows > 1 && y_stride < w->rows && y_stride > -(int64_t)w->rows) return AWSRC_ERR_INVALID_ARG;
  if ((s = check_workspace(workspace, workspace_bytes)) != AWSRC_OK) return s;
  // tiles are numbered in 32 bits
  if ((int64_t)a.w.tiles() * ((a.x.rows + 15) / 16) > INT_MAX / 2) return AWSRC_ERR_UNSUPPORTED;
  a.y = y;
  a.ys = y_stride;
  a.y_f32 = y_dtype == AWSRC_DTYPE_F32;
  a.status = static_cast<uint32_t*>(workspace);
  a.wait_ns = wait_limit_ns();
  a.stall = wait_test_stall();
  *out = a;
  return AWSRC_OK;
}

}  // namespace

}  // namespace awsrc

using namespace awsrc;

extern "C" {

awsrc_status awsrc_step_workspace_bytes(size_t* bytes) {
  if (!bytes) return AWSRC_ERR_INVALID_ARG;
  *bytes = kStepWorkspace;
  return AWSRC_OK;
}

awsrc_status awsrc_step_workspace_init(void* workspace, size_t workspace_bytes, void* stream) {
  const awsrc_status s = check_workspace(workspace, workspace_bytes);
  if (s != AWSRC_OK) return s;
  const cudaError_t e = cudaMemsetAsync(workspace, 0, kStepWorkspace, (cudaStream_t)stream);
  return e == cudaSuccess ? AWSRC_OK : cuda_fail(e, "step_workspace_init");
}

awsrc_status awsrc_kv_plan(const awsrc_kv_pool* pool, const int32_t* keep, const int32_t* add, int32_t n_tok,
                           int32_t* q_start, int32_t* tok_seq, int32_t* tok_pos, int64_t* tok_slot, void* workspace,
                           size_t workspace_bytes, void* stream) {
  if (!pool || pool->n_pages < 1 || pool->n_seq < 0 || pool->table_stride < 1 || n_tok < 0) return AWSRC_ERR_INVALID_ARG;
  if (pool->page != 16 && pool->page != 32 && pool->page != 64 && pool->page != 128) return AWSRC_ERR_SHAPE;
  if (pool->n_seq > kPlanMaxSeq || pool->n_pages > (1 << 30) || n_tok > (1 << 30) ||
      (int64_t)pool->table_stride * pool->page > (1 << 30)) return AWSRC_ERR_UNSUPPORTED;
  if (!pool->page_table || !pool->kv_len || !pool->free_pages || !pool->free_count || !add || !q_start)
    return AWSRC_ERR_INVALID_ARG;
  for (const void* p : {(const void*)pool->page_table, (const void*)pool->kv_len, (const void*)pool->free_pages,
                        (const void*)pool->free_count, (const void*)keep, (const void*)add, (const void*)q_start,
                        (const void*)tok_seq, (const void*)tok_pos})
    if (!aligned(p, 4)) return AWSRC_ERR_INVALID_ARG;
  if (!aligned(tok_slot, 8)) return AWSRC_ERR_INVALID_ARG;
  const awsrc_status s = check_workspace(workspace, workspace_bytes);
  if (s != AWSRC_OK) return s;
  if (keep == pool->kv_len) return AWSRC_ERR_INVALID_ARG;  // what was held would be lost: its pages never came back
  PlanArgs a{pool->n_pages, pool->page, 4, pool->n_seq, pool->table_stride, n_tok, pool->page_table, pool->kv_len,
             pool->free_pages, pool->free_count, keep, add, q_start, tok_seq, tok_pos, tok_slot,
             static_cast<uint32_t*>(workspace), static_cast<uint32_t*>(workspace) + kArrivedAt, 0};
  while ((1 << a.log_page) < a.page) ++a.log_page;
  const cudaError_t e = launch_plan(a, (cudaStream_t)stream);
  return e == cudaSuccess ? AWSRC_OK : cuda_fail(e, "kv_plan");
}

awsrc_status awsrc_verify_drafts(int32_t n_seq, int32_t n_rows, int32_t vocab, int32_t max_draft, const int32_t* row_start,
                                 const int32_t* ids, const awsrc_probs* target, const awsrc_probs* draft, const float* u,
                                 const float* r, const int32_t* kv_len, int32_t* accepted, int32_t* tokens, int32_t* keep,
                                 void* workspace, size_t workspace_bytes, void* stream) {
  if (n_seq < 0 || n_rows < 0 || max_draft < 0) return AWSRC_ERR_INVALID_ARG;
  if (vocab < 1) return AWSRC_ERR_SHAPE;
  if (n_seq > 65535 || vocab > (1 << 18) || max_draft > (1 << 20)) return AWSRC_ERR_UNSUPPORTED;
  if (!row_start || !ids || !target || !u || !r || !accepted || !tokens || !kv_len != !keep) return AWSRC_ERR_INVALID_ARG;
  awsrc_status s = check_rows(target->p, target->dtype);
  if (s != AWSRC_OK || (draft && (s = check_rows(draft->p, draft->dtype)) != AWSRC_OK)) return s;
  for (const void* p : {(const void*)row_start, (const void*)ids, (const void*)u, (const void*)r, (const void*)kv_len,
                        (const void*)accepted, (const void*)tokens, (const void*)keep})
    if (!aligned(p, 4)) return AWSRC_ERR_INVALID_ARG;
  if ((s = check_workspace(workspace, workspace_bytes)) != AWSRC_OK) return s;
  if (n_seq == 0) return AWSRC_OK;
  const VerifyArgs a{n_seq, n_rows, vocab, max_draft, row_start, ids, target->p, draft ? draft->p : nullptr, target->stride,
                     draft ? draft->stride : 0, u, r, kv_len, accepted, tokens, keep, static_cast<uint32_t*>(workspace)};
  const cudaError_t e = launch_verify(a, target->dtype, draft ? draft->dtype : AWSRC_DTYPE_F32, (cudaStream_t)stream);
  return e == cudaSuccess ? AWSRC_OK : cuda_fail(e, "verify_drafts");
}

awsrc_status awsrc_fp8_matrix_bytes(int32_t rows, int32_t cols, size_t* codes, size_t* exps) {
  if (!codes || !exps) return AWSRC_ERR_INVALID_ARG;
  const awsrc_fp8_matrix m{rows, cols, nullptr, nullptr};
  Fp8Mat f;
  const awsrc_status s = check_matrix(&m, false, &f);
  if (s != AWSRC_OK) return s;
  *codes = codes_bytes(f);
  *exps = exps_bytes(f);
  return AWSRC_OK;
}

awsrc_status awsrc_fp8_quantize(const void* x, int32_t dtype, int64_t stride, const awsrc_fp8_matrix* out, void* stream) {
  Fp8Mat m;
  awsrc_status s = check_matrix(out, true, &m);
  if (s != AWSRC_OK || (s = check_rows(x, dtype)) != AWSRC_OK) return s;
  if (m.rows == 0) return AWSRC_OK;
  const cudaError_t e = launch_fp8_quantize(x, dtype, stride, m, (cudaStream_t)stream);
  return e == cudaSuccess ? AWSRC_OK : cuda_fail(e, "fp8_quantize");
}

awsrc_status awsrc_fp8_gemm(const awsrc_fp8_matrix* x, const awsrc_fp8_matrix* w, void* y, int32_t y_dtype, int64_t y_stride,
                            void* workspace, size_t workspace_bytes, void* stream) {
  GemmArgs a;
  const awsrc_status s = gemm_args(x, w, y, y_dtype, y_stride, workspace, workspace_bytes, &a);
  if (s != AWSRC_OK) return s;
  if (a.x.rows == 0 || a.w.rows == 0) return AWSRC_OK;
  const cudaError_t e = launch_fp8_gemm(a, (cudaStream_t)stream);
  return e == cudaSuccess ? AWSRC_OK : cuda_fail(e, "fp8_gemm");
}

awsrc_status awsrc_fp8_linear(const void* x, int32_t x_dtype, int64_t x_stride, const awsrc_fp8_matrix* x8,
                              const awsrc_fp8_matrix* w, void* y, int32_t y_dtype, int64_t y_stride, void* workspace,
                              size_t workspace_bytes, void* stream) {
  GemmArgs a;
  awsrc_status s = gemm_args(x8, w, y, y_dtype, y_stride, workspace, workspace_bytes, &a);
  if (s != AWSRC_OK || (s = check_rows(x, x_dtype)) != AWSRC_OK) return s;
  if (x8->codes == w->codes || x8->exps == w->exps || share(a.x, a.w)) return AWSRC_ERR_INVALID_ARG;
  if (a.x.rows == 0) return AWSRC_OK;
  if (a.w.rows == 0) return awsrc_fp8_quantize(x, x_dtype, x_stride, x8, stream);  // x8 is written all the same
  // few rows of x are read while others' results are written
  const int64_t xs = size_of(x_dtype), ys = size_of(y_dtype);
  if (share(Rows{x, x_stride * xs, a.x.cols * xs}, Rows{y, y_stride * ys, a.w.rows * ys}, a.x.rows)) return AWSRC_ERR_INVALID_ARG;
  bool itself;
  cudaError_t e = fp8_gemm_quantizes(a, x_dtype == AWSRC_DTYPE_BF16, &itself);
  if (e == cudaSuccess && itself) {
    a.raw = x;
    a.raw_stride = x_stride;
    a.raw_bf16 = x_dtype == AWSRC_DTYPE_BF16;
  } else if (e == cudaSuccess) {
    // the quantising kernel lets the product start only after it has waited for all kernels before it
    a.early = 1;
    e = launch_fp8_quantize(x, x_dtype, x_stride, a.x, (cudaStream_t)stream);
  }
  if (e == cudaSuccess) e = launch_fp8_gemm(a, (cudaStream_t)stream);
  return e == cudaSuccess ? AWSRC_OK : cuda_fail(e, "fp8_linear");
}

}  // extern "C"
