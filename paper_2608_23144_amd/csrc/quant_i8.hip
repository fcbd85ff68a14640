// Rows of floating values as int8 codes with one fp32 scale per row: the
// activations of an int8 linear layer (one scale per token) and its weights
// (one per output channel).
//
// Built without FMA contraction: scale, inverse and codes are single fp32
// operations, so that the codes are the recipe's to the bit.
#include "serve_internal.h"

namespace awsrc {

namespace {

__device__ __forceinline__ void store8(int8_t* __restrict__ c, uint2 w, int64_t n, bool wide) {
  if (wide && n >= 8) {
    *reinterpret_cast<uint2*>(c) = w;
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < n) c[e] = (int8_t)((e < 4 ? w.x : w.y) >> (8 * (e & 3)));
  }
}

// WPR wavefronts per row, CH pieces of 8 values per lane in registers, so
// that a row is read once; WPR = 1 takes four rows per workgroup.
template <typename T, int WPR, int CH>
__global__ __launch_bounds__(64 * (WPR == 1 ? 4 : WPR)) void k_quantize_rows(const T* __restrict__ X, int64_t rows, int64_t cols,
                                                                             int64_t ldx, int8_t* __restrict__ codes,
                                                                             int64_t ldc, int64_t pad, float* __restrict__ scale,
                                                                             bool wide_x, bool wide_c) {
  __shared__ float part[WPR];
  const int wave = threadIdx.x >> 6;
  const int64_t wg = workgroup<64 * (WPR == 1 ? 4 : WPR)>();
  const int64_t row = WPR == 1 ? wg * 4 + wave : wg;
  if (row >= rows) return;
  const int t = WPR == 1 ? (threadIdx.x & 63) : threadIdx.x;
  const T* x = X + row * ldx;
  // Where rows do not lie on 16 bytes a lane takes every (64 WPR)-th value of a
  // stretch instead of eight adjacent ones, so that a load still reads whole lines.
  const int64_t step = wide_x ? 1 : WPR * 64;
  const auto start = [&](int i) { return wide_x ? (int64_t)(i * WPR * 64 + t) * 8 : (int64_t)i * WPR * 512 + t; };
  float v[CH][8];
  float m = 0.0f;
#pragma unroll
  for (int i = 0; i < CH; ++i) {
    const int64_t at = start(i);
    if (wide_x) {
      load8(x + at, cols - at, true, v[i]);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[i][e] = at + e * step < cols ? to_f32(x[at + e * step]) : 0.0f;
    }
  }
#pragma unroll
  for (int i = 0; i < CH; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) m = amax_keep(m, v[i][e]);
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) m = amax_keep(m, __shfl_xor(m, off, 64));
  if constexpr (WPR > 1) {
    if ((t & 63) == 0) part[wave] = m;
    __syncthreads();
    m = part[0];
#pragma unroll
    for (int w = 1; w < WPR; ++w) m = amax_keep(m, part[w]);
  }
  const float s = scale_of_amax(m);
  const float inv = inverse_scale(s);
  const bool live = s == s;
  int8_t* c = codes + row * ldc;
#pragma unroll
  for (int i = 0; i < CH; ++i) {
    const int64_t at = start(i);
    if (at >= pad) continue;
    const uint2 w = codes8(v[i], inv, live);
    if (wide_x) {
      store8(c + at, w, pad - at, wide_c);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (at + e * step < pad) c[at + e * step] = (int8_t)((e < 4 ? w.x : w.y) >> (8 * (e & 3)));
    }
  }
  if (t == 0) scale[row] = s;
}

// Rows longer than the registers take: read twice, the second time mostly from the caches.
template <typename T>
__global__ __launch_bounds__(1024) void k_quantize_long_rows(const T* __restrict__ X, int64_t rows, int64_t cols, int64_t ldx,
                                                             int8_t* __restrict__ codes, int64_t ldc, int64_t pad,
                                                             float* __restrict__ scale, bool wide_x, bool wide_c) {
  __shared__ float part[16];
  const int64_t row = workgroup<1024>();
  if (row >= rows) return;
  const T* x = X + row * ldx;
  int8_t* c = codes + row * ldc;
  float m = 0.0f;
  for (int64_t at = (int64_t)threadIdx.x * 8; at < cols; at += 8192) {
    float v[8];
    load8(x + at, cols - at, wide_x, v);
#pragma unroll
    for (int e = 0; e < 8; ++e) m = amax_keep(m, v[e]);
  }
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) m = amax_keep(m, __shfl_xor(m, off, 64));
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = m;
  __syncthreads();
  m = part[0];
#pragma unroll
  for (int w = 1; w < 16; ++w) m = amax_keep(m, part[w]);
  const float s = scale_of_amax(m);
  const float inv = inverse_scale(s);
  for (int64_t at = (int64_t)threadIdx.x * 8; at < pad; at += 8192) {
    float v[8];
    load8(x + at, cols - at, wide_x, v);
    store8(c + at, codes8(v, inv, s == s), pad - at, wide_c);
  }
  if (threadIdx.x == 0) scale[row] = s;
}

template <typename T>
hipError_t launch(const void* X, int64_t rows, int64_t cols, int64_t ldx, int8_t* codes, int64_t ldc, float* scale,
                  hipStream_t st) {
  const T* x = static_cast<const T*>(X);
  // Zeros up to the next 16 bytes only where rows lie on 16 bytes, as the products take them: the fill then ends inside the
  // row's own stride.  Of a column slice that starts anywhere else it would reach into the next columns or the next row.
  const bool on16 = ((reinterpret_cast<uintptr_t>(codes) | (uintptr_t)ldc) & 15) == 0;
  const int64_t pad = on16 ? (cols + 15) / 16 * 16 : cols;
  const bool wx = ((reinterpret_cast<uintptr_t>(X) | (uintptr_t)(ldx * sizeof(T))) & 15) == 0;
  const bool wc = ((reinterpret_cast<uintptr_t>(codes) | (uintptr_t)ldc) & 7) == 0;
#define AWSRC_ROWS(WPR, CH)                                                                                            \
  hipLaunchKernelGGL((k_quantize_rows<T, WPR, CH>),                                                                    \
                     grid_of<64 * (WPR == 1 ? 4 : WPR)>(WPR == 1 ? (rows + 3) / 4 : rows),                            \
                     dim3(64 * (WPR == 1 ? 4 : WPR)), 0, st, x, rows, cols, ldx, codes, ldc, pad, scale, wx, wc)
  // One wavefront a row where there are rows enough to fill the machine and a
  // row fits its registers; else as many as leave each lane one or two pieces,
  // since a call of few rows waits for memory, not on bandwidth (bf16, in us:
  // 1 x 5120 3.0 with sixteen wavefronts, 3.8 with four; 8192 x 2048 13.0 with one,
  // 19.4 with four; 8192 x 5120 30, 4.1 TB/s; 8192 x 11008 57 with eight, 73 with sixteen).
  if (cols <= 512) AWSRC_ROWS(1, 1);
  else if (rows >= 2048 && cols <= 2048) AWSRC_ROWS(1, 4);
  else if (cols <= 2048) AWSRC_ROWS(4, 1);
  else if (rows >= 1024 && cols <= 8192) AWSRC_ROWS(4, 4);
  else if (cols <= 8192) AWSRC_ROWS(16, 1);
  else if (rows >= 1024 && cols <= 12288) AWSRC_ROWS(8, 3);
  else if (cols <= 16384) AWSRC_ROWS(16, 2);
  else
    hipLaunchKernelGGL((k_quantize_long_rows<T>), grid_of<1024>(rows), dim3(1024), 0, st, x, rows, cols, ldx, codes, ldc,
                       pad, scale, wx, wc);
#undef AWSRC_ROWS
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
