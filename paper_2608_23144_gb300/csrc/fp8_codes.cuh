// fp8_codes.cuh — a warp's 128 columns of a row to e4m3 codes with one power-of-two scale.
#pragma once

#include "kv_paged.cuh"

namespace awsrc {
namespace fp8 {

constexpr int kExpLeast = -64;

// Smallest e with amax <= 448 * 2^e (448 = 1.75 * 2^8), at least kExpLeast.
__device__ __forceinline__ int exponent_of(float amax) {
  const uint32_t u = __float_as_uint(amax);
  return max((int)(u >> 23) - 127 - 8 + ((u & 0x7FFFFFu) > 0x600000u ? 1 : 0), kExpLeast);
}

template <bool kVec>
__device__ __forceinline__ void load4(const float* p, int have, float* v) {
  if (kVec && have >= 4) {
    const float4 x = __ldcg(reinterpret_cast<const float4*>(p));
    v[0] = x.x, v[1] = x.y, v[2] = x.z, v[3] = x.w;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = i < have ? p[i] : 0.0f;
  }
}
template <bool kVec>
__device__ __forceinline__ void load4(const __nv_bfloat16* p, int have, float* v) {
  if (kVec && have >= 4) {
    const uint2 x = __ldcg(reinterpret_cast<const uint2*>(p));
    v[0] = __uint_as_float(x.x << 16), v[1] = __uint_as_float(x.x & 0xFFFF0000u);
    v[2] = __uint_as_float(x.y << 16), v[3] = __uint_as_float(x.y & 0xFFFF0000u);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = i < have ? __bfloat162float(p[i]) : 0.0f;
  }
}

// The lane's 4 codes and the block's exponent + 127 of 128 columns, 4 a lane; `have` of
// the lane's columns exist. A block that is not finite: NaN codes, exponent 0.
struct Codes4 {
  uint32_t codes, biased;
};
__device__ __forceinline__ Codes4 codes_of(const float* v, int have) {
  float amax = 0.0f;
#pragma unroll
  for (int j = 0; j < 4; ++j) amax = fmax_nan(amax, fabsf(v[j]));
  // magnitudes as integers keep their order, infinity and NaN above all
  const uint32_t most = __reduce_max_sync(0xffffffffu, __float_as_uint(amax));
  if (most >= 0x7F800000u) return Codes4{have >= 4 ? 0x7F7F7F7Fu : have > 0 ? 0x7F7F7F7Fu >> (32 - 8 * have) : 0u, 127u};
  const int e = exponent_of(__uint_as_float(most));
  const float s = __int_as_float((127 - e) << 23);
  return Codes4{e4m3x2(__fmul_rn(v[0], s), __fmul_rn(v[1], s)) | e4m3x2(__fmul_rn(v[2], s), __fmul_rn(v[3], s)) << 16,
                (uint32_t)(e + 127)};
}

}  // namespace fp8
}  // namespace awsrc
