// fp8_quantize.cu — rows to e4m3 codes with one power-of-two scale per row and 128
// columns, in the byte order the tensor cores read (include/awsrc.h).
//
// One pass: a warp holds 4 blocks of a row in registers, finds each block's
// largest magnitude over the warp and writes the codes; its 4 exponents are one
// word of the scale layout. Floor: the rows read, the codes written, once.
#include "internal.h"
#include "kv_paged.cuh"
#include "step.cuh"

namespace awsrc {

namespace {

constexpr int kWarps = 8;  // rows of a thread block
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

template <typename T, bool kVec>
__global__ void __launch_bounds__(32 * kWarps) fp8_quantize_kernel(const T* x, int64_t stride, const __grid_constant__ Fp8Mat m) {
  step_wait();
  step_trigger();
  const int lane = threadIdx.x & 31, r = blockIdx.x * kWarps + (threadIdx.x >> 5);
  const int g = blockIdx.y;  // 4 blocks of 128 columns
  if (r >= m.rows) return;
  const int n = min(4, m.blocks() - 4 * g);
  const T* p = x + (int64_t)r * stride + 512ll * g + 4 * lane;
  float v[4][4];
#pragma unroll
  for (int i = 0; i < 4; ++i) load4<kVec>(p + 128 * i, m.cols - (512 * g + 128 * i + 4 * lane), v[i]);
  const int64_t rows8 = m.rows8();
  uint8_t* out = m.codes + (4ll * g * rows8 + r) * 128 + 16 * ((lane >> 2) ^ (r & 7)) + 4 * (lane & 3);
  uint32_t exps = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float amax = 0.0f;
#pragma unroll
    for (int j = 0; j < 4; ++j) amax = fmax_nan(amax, fabsf(v[i][j]));
    // magnitudes as integers keep their order, infinity and NaN above all
    const uint32_t most = __reduce_max_sync(0xffffffffu, __float_as_uint(amax));
    const int have = m.cols - (512 * g + 128 * i + 4 * lane);  // columns past the last are 0 in any block
    uint32_t codes = have >= 4 ? 0x7F7F7F7Fu : have > 0 ? 0x7F7F7F7Fu >> (32 - 8 * have) : 0u;
    int e = 0;
    if (most < 0x7F800000u) {
      e = exponent_of(__uint_as_float(most));
      const float s = __int_as_float((127 - e) << 23);
      codes = e4m3x2(__fmul_rn(v[i][0], s), __fmul_rn(v[i][1], s)) |
              e4m3x2(__fmul_rn(v[i][2], s), __fmul_rn(v[i][3], s)) << 16;
    }
    if (i < n) {
      *reinterpret_cast<uint32_t*>(out + i * rows8 * 128) = codes;
      exps |= (uint32_t)(e + 127) << (8 * i);
    }
  }
  if (lane == 0)
    *reinterpret_cast<uint32_t*>(m.exps + ((int64_t)g * m.tiles() + (r >> 7)) * 512 + (r & 31) * 16 + ((r & 127) >> 5) * 4) = exps;
}

template <typename T>
cudaError_t launch(const void* x, int64_t stride, const Fp8Mat& m, cudaStream_t st) {
  const dim3 grid((m.rows + kWarps - 1) / kWarps, (m.blocks() + 3) / 4);
  const bool vec = (reinterpret_cast<uintptr_t>(x) | (uintptr_t)(stride * (int64_t)sizeof(T))) % (4 * sizeof(T)) == 0;
  const T* p = static_cast<const T*>(x);
  return vec ? launch_step(fp8_quantize_kernel<T, true>, grid, 32 * kWarps, 0, 1, st, p, stride, m)
             : launch_step(fp8_quantize_kernel<T, false>, grid, 32 * kWarps, 0, 1, st, p, stride, m);
}

}  // namespace

cudaError_t launch_fp8_quantize(const void* x, int dtype, int64_t stride, const Fp8Mat& m, cudaStream_t st) {
  const cudaError_t e = dtype == AWSRC_DTYPE_BF16 ? launch<__nv_bfloat16>(x, stride, m, st) : launch<float>(x, stride, m, st);
  if (e != cudaSuccess) return e;
  note_launches(1);
  return cudaGetLastError();
}

}  // namespace awsrc
