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
  const int q0 = __ldg(a.q_start + b), q1 = __ldg(a.q_start + b + 1), kv = __ldg(a.kv_len + b);
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

// Attention: thread blocks a launch may have (two per SM), each with two slots
// for partial results of the first and last tile it shares with others.
constexpr int kMaxAttnBlocks = 304;
constexpr int kSlotRows = 64;

struct AttnArgs {
  KvArgs c;
  KvRows q, out;
  float* lse;
  float score_mul;  // sm_scale log2(e)
  int causal;
  int min_units;    // least share of a block
  int* arrived;     // per block: arrivals at the shared tile that begins in its share
  float* partial;
  int64_t slot_floats;
};

// Row tiles a batch can have at most.
inline int64_t tiles_upper(const KvArgs& c, int tile_rows) {
  return (int64_t)c.n_tok * c.group / tile_rows + (c.n_seq < c.n_tok ? c.n_seq : c.n_tok);
}

cudaError_t launch_kv_append(const KvArgs& c, int head_dim, int dtype, const KvRows& q, const KvRows& k,
                             const KvRows& v, const KvRows& qo, const float* cos, const float* sin, int rope_rows,
                             int rotary_dim, int interleaved, cudaStream_t st);
cudaError_t launch_paged_rows(const AttnArgs& a, int head_dim, int dtype, int max_new, int max_kv, cudaStream_t st);

}  // namespace awsrc
