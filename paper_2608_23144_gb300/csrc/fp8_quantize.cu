// fp8_quantize.cu — rows to e4m3 codes with one power-of-two scale per row and 128
// columns, in the byte order the tensor cores read (include/awsrc.h).
//
// One pass: a warp holds 4 blocks of a row in registers, finds each block's
// largest magnitude over the warp and writes the codes; its 4 exponents are one
// word of the scale layout. Floor: the rows read, the codes written, once.
// Measured, rows from memory: 11008 x 2048 float32 17.4 us, 6.5 TB/s or 96% of the measured
// copy (an odd stride, loads of one element, 19.0); 1023 x 3584 bf16 4.6 us (floor 1.6; out
// of the L2 3.0), the latency of one round of loads; 8192 x 3584 bf16 22 to 28 (floor 13):
// a warp has half the bytes in flight there that it has in float32.
#include "fp8_codes.cuh"
#include "internal.h"
#include "step.cuh"

namespace awsrc {

namespace {

using namespace fp8;

constexpr int kWarps = 8;  // rows of a thread block
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
    const Codes4 c = codes_of(v[i], m.cols - (512 * g + 128 * i + 4 * lane));
    if (i < n) {
      *reinterpret_cast<uint32_t*>(out + i * rows8 * 128) = c.codes;
      exps |= c.biased << (8 * i);
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
