// Rows of floating values as int8 codes with one fp32 scale per row: the
// activations of an int8 linear layer (one scale per token) and its weights
// (one per output channel).
//
// Built without FMA contraction: scale, inverse and codes are single fp32
// operations, so that the codes are the recipe's to the bit.
#include "serve_internal.h"

namespace awsrc {

namespace {

template <typename T>
__global__ __launch_bounds__(256) void k_quantize_rows(const T* __restrict__ X, int64_t cols, int64_t ldx,
                                                       int8_t* __restrict__ codes, int64_t ldc, int64_t pad,
                                                       float* __restrict__ scale) {
  __shared__ float part[4];
  const int64_t row = blockIdx.x;
  const T* x = X + row * ldx;
  int8_t* c = codes + row * ldc;
  float m = 0.0f;
  for (int64_t i = threadIdx.x; i < cols; i += 256) m = amax_keep(m, to_f32(x[i]));
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) m = amax_keep(m, __shfl_xor(m, off, 64));
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = m;
  __syncthreads();
  m = part[0];
#pragma unroll
  for (int w = 1; w < 4; ++w) m = amax_keep(m, part[w]);
  const float s = scale_of_amax(m);
  const float inv = inverse_scale(s);
  for (int64_t i = threadIdx.x; i < pad; i += 256) c[i] = i < cols ? (int8_t)code_of(to_f32(x[i]), inv) : (int8_t)0;
  if (threadIdx.x == 0) scale[row] = s;
}

template <typename T>
hipError_t launch(const void* X, int64_t rows, int64_t cols, int64_t ldx, int8_t* codes, int64_t ldc, float* scale,
                  hipStream_t st) {
  int64_t pad = (cols + 15) / 16 * 16;
  if (pad > ldc) pad = ldc;
  hipLaunchKernelGGL((k_quantize_rows<T>), dim3((unsigned)rows), dim3(256), 0, st, static_cast<const T*>(X), cols, ldx,
                     codes, ldc, pad, scale);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_quantize_rows(const void* X, int x_dtype, int64_t rows, int64_t cols, int64_t ldx, int8_t* codes,
                                int64_t ldc, float* scale, hipStream_t st) {
  if (x_dtype == AWSRC_DTYPE_F32) return launch<float>(X, rows, cols, ldx, codes, ldc, scale, st);
  if (x_dtype == AWSRC_DTYPE_BF16) return launch<__bf16>(X, rows, cols, ldx, codes, ldc, scale, st);
  return launch<_Float16>(X, rows, cols, ldx, codes, ldc, scale, st);
}

}  // namespace awsrc
