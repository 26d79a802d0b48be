// api_kv.cu — the extern "C" entry points of the paged 8-bit cache declared in
// include/awsrc.h: argument validation, workspace layout, launches.
#include <climits>
#include <cmath>

#include "internal.h"
#include "kv_paged.cuh"

namespace awsrc {

namespace {

bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

awsrc_status check_cache(const awsrc_kv_cache* c, int32_t n_heads, bool pointers) {
  if (!c || c->n_pages < 1 || c->n_kv_heads < 1 || n_heads < 1) return AWSRC_ERR_INVALID_ARG;
  if (c->page != 16 && c->page != 32 && c->page != 64 && c->page != 128) return AWSRC_ERR_SHAPE;
  if (c->head_dim != 64 && c->head_dim != 128) return AWSRC_ERR_SHAPE;
  if (n_heads % c->n_kv_heads != 0) return AWSRC_ERR_SHAPE;
  if (n_heads / c->n_kv_heads > 1024) return AWSRC_ERR_UNSUPPORTED;
  if (pointers && (!c->k || !c->v || !c->k_exp || !c->v_exp || !aligned(c->k, 16) || !aligned(c->v, 16)))
    return AWSRC_ERR_INVALID_ARG;
  return AWSRC_OK;
}

struct AttnLayout {
  size_t arrived, shared, partial, total;
  int64_t row_slot, tile_slot;  // floats of a partial result of either kernel
};

AttnLayout attn_layout(const awsrc_kv_cache& c) {
  AttnLayout L{};
  L.arrived = kStatusBytes;
  const size_t blocks = max_attn_blocks(c.head_dim);
  L.shared = L.arrived + align_up(blocks * sizeof(int), 256);
  L.partial = L.shared + align_up(blocks * sizeof(SharedTile), 256);
  L.row_slot = (int64_t)kSlotRows * (c.head_dim + 2);
  L.tile_slot = (int64_t)kTileSlotRows * (c.head_dim + 2);
  const size_t rows = 2 * blocks * L.row_slot, tiles = (size_t)2 * kMaxTileBlocks * L.tile_slot;
  L.total = L.partial + align_up((rows > tiles ? rows : tiles) * sizeof(float), 256);
  return L;
}

// Cache, batch and workspace of a call -> what the kernels take.
awsrc_status kv_args(const awsrc_kv_cache* c, const awsrc_kv_batch* b, int32_t n_heads, void* workspace,
                     size_t workspace_bytes, KvArgs* out) {
  awsrc_status s = check_cache(c, n_heads, true);
  if (s != AWSRC_OK) return s;
  if (!b || b->n_seq < 0 || b->n_tok < 0 || b->max_new < 0 || b->max_kv < 0 || b->table_stride < 1)
    return AWSRC_ERR_INVALID_ARG;
  if (!b->q_start || !b->kv_len || !b->page_table || !aligned(b->q_start, 4) || !aligned(b->kv_len, 4) ||
      !aligned(b->page_table, 4))
    return AWSRC_ERR_INVALID_ARG;
  // positions and rows are 32-bit in the kernels
  if ((int64_t)b->table_stride * c->page > (1 << 30) || (int64_t)b->n_tok * n_heads > INT_MAX)
    return AWSRC_ERR_UNSUPPORTED;
  if (!workspace || workspace_bytes < attn_layout(*c).total) return AWSRC_ERR_WORKSPACE;
  if (!aligned(workspace, 256)) return AWSRC_ERR_INVALID_ARG;
  KvArgs a{};
  a.k = c->k;
  a.v = c->v;
  a.k_exp = c->k_exp;
  a.v_exp = c->v_exp;
  a.n_pages = c->n_pages;
  a.page = c->page;
  for (a.log_page = 4; (1 << a.log_page) < c->page;) ++a.log_page;
  a.kv_heads = c->n_kv_heads;
  a.n_heads = n_heads;
  a.group = n_heads / c->n_kv_heads;
  a.n_seq = b->n_seq;
  a.n_tok = b->n_tok;
  a.table_stride = b->table_stride;
  a.q_start = b->q_start;
  a.kv_len = b->kv_len;
  a.table = b->page_table;
  a.status = static_cast<uint32_t*>(workspace);
  *out = a;
  return AWSRC_OK;
}

awsrc_status kv_rows(const awsrc_rows* r, int32_t dtype, KvRows* out) {
  if (!r || !r->p || r->dtype != dtype) return AWSRC_ERR_INVALID_ARG;
  if (!aligned(r->p, dtype == AWSRC_DTYPE_BF16 ? 2 : 4)) return AWSRC_ERR_INVALID_ARG;
  *out = KvRows{r->p, r->tok_stride, r->head_stride};
  return AWSRC_OK;
}

bool is_dtype(const awsrc_rows* r) { return r && (r->dtype == AWSRC_DTYPE_F32 || r->dtype == AWSRC_DTYPE_BF16); }

}  // namespace

}  // namespace awsrc

using namespace awsrc;

extern "C" {

awsrc_status awsrc_attention_workspace_bytes(const awsrc_kv_cache* cache, int32_t n_heads, size_t* bytes) {
  if (!bytes) return AWSRC_ERR_INVALID_ARG;
  const awsrc_status s = check_cache(cache, n_heads, false);
  if (s != AWSRC_OK) return s;
  *bytes = attn_layout(*cache).total;
  return AWSRC_OK;
}

awsrc_status awsrc_attention_workspace_init(const awsrc_kv_cache* cache, int32_t n_heads, void* workspace,
                                            size_t workspace_bytes, void* stream) {
  const awsrc_status s = check_cache(cache, n_heads, false);
  if (s != AWSRC_OK) return s;
  const AttnLayout L = attn_layout(*cache);
  if (!workspace || workspace_bytes < L.total) return AWSRC_ERR_WORKSPACE;
  if (!aligned(workspace, 256)) return AWSRC_ERR_INVALID_ARG;
  const cudaError_t e = cudaMemsetAsync(workspace, 0, L.partial, (cudaStream_t)stream);
  return e == cudaSuccess ? AWSRC_OK : cuda_fail(e, "attention_workspace_init");
}

awsrc_status awsrc_kv_append(const awsrc_kv_cache* cache, const awsrc_kv_batch* batch, int32_t n_heads,
                             const awsrc_rows* q, const awsrc_rows* k, const awsrc_rows* v,
                             const awsrc_rows* q_out, const float* cos, const float* sin, int32_t rope_rows,
                             int32_t rotary_dim, int32_t interleaved, void* workspace, size_t workspace_bytes,
                             void* stream) {
  KvArgs a;
  awsrc_status s = kv_args(cache, batch, n_heads, workspace, workspace_bytes, &a);
  if (s != AWSRC_OK) return s;
  if (!is_dtype(q)) return AWSRC_ERR_INVALID_ARG;
  KvRows rq, rk, rv, ro;
  if ((s = kv_rows(q, q->dtype, &rq)) != AWSRC_OK || (s = kv_rows(k, q->dtype, &rk)) != AWSRC_OK ||
      (s = kv_rows(v, q->dtype, &rv)) != AWSRC_OK || (s = kv_rows(q_out, q->dtype, &ro)) != AWSRC_OK)
    return s;
  if (rotary_dim < 0 || rotary_dim > cache->head_dim || rotary_dim % 2 != 0) return AWSRC_ERR_SHAPE;
  if (interleaved != 0 && interleaved != 1) return AWSRC_ERR_INVALID_ARG;
  if (rotary_dim > 0 && (!cos || !sin || rope_rows < 1 || !aligned(cos, 4) || !aligned(sin, 4)))
    return AWSRC_ERR_INVALID_ARG;
  if (a.n_tok == 0 || a.n_seq == 0) return AWSRC_OK;
  const cudaError_t e = launch_kv_append(a, cache->head_dim, q->dtype, rq, rk, rv, ro, cos, sin, rope_rows, rotary_dim,
                                         interleaved, (cudaStream_t)stream);
  return e == cudaSuccess ? AWSRC_OK : cuda_fail(e, "kv_append");
}

awsrc_status awsrc_paged_attention(const awsrc_kv_cache* cache, const awsrc_kv_batch* batch, int32_t n_heads,
                                   const awsrc_rows* q, const awsrc_rows* out, float* lse, float sm_scale,
                                   int32_t causal, void* workspace, size_t workspace_bytes, void* stream) {
  AttnArgs a{};
  awsrc_status s = kv_args(cache, batch, n_heads, workspace, workspace_bytes, &a.c);
  if (s != AWSRC_OK) return s;
  if (!is_dtype(q)) return AWSRC_ERR_INVALID_ARG;
  if ((s = kv_rows(q, q->dtype, &a.q)) != AWSRC_OK || (s = kv_rows(out, q->dtype, &a.out)) != AWSRC_OK) return s;
  if (!aligned(lse, 4) || !std::isfinite(sm_scale) || (causal != 0 && causal != 1)) return AWSRC_ERR_INVALID_ARG;
  if (a.c.n_tok == 0 || a.c.n_seq == 0) return AWSRC_OK;
  const AttnLayout L = attn_layout(*cache);
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  a.lse = lse;
  a.score_mul = sm_scale * 1.4426950408889634f;
  a.causal = causal;
  a.arrived = reinterpret_cast<int*>(ws + L.arrived);
  a.shared = reinterpret_cast<SharedTile*>(ws + L.shared);
  a.partial = reinterpret_cast<float*>(ws + L.partial);
  a.wait_ns = wait_limit_ns();
  a.stall = wait_test_stall();
  // BF16 with more rows per kv head than the row kernel takes in one warp tile
  // goes to the tensor-memory kernel, which reads and writes rows in vectors
  const bool tiles = q->dtype == AWSRC_DTYPE_BF16 && (int64_t)batch->max_new * a.c.group > 16 &&
                     rows_aligned(a.q, 2) && rows_aligned(a.out, 2);
  a.slot_floats = tiles ? L.tile_slot : L.row_slot;
  const cudaError_t e = tiles ? launch_paged_tiles(a, cache->head_dim, batch->max_kv, (cudaStream_t)stream)
                              : launch_paged_rows(a, cache->head_dim, q->dtype, batch->max_new, batch->max_kv,
                                                  (cudaStream_t)stream);
  return e == cudaSuccess ? AWSRC_OK : cuda_fail(e, "paged_attention");
}

}  // extern "C"
