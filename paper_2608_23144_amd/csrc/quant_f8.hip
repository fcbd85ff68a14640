// Matrices as e4m3 codes with one fp32 scale for each block of 1 x 128 values
// (activations) or 128 x 128 (weights), and back.
//
// Built without FMA contraction: scale, inverse and codes are single fp32
// operations, so that the codes are the recipe's to the bit.
//
// Bound by memory: every value is read once and kept in registers between its block's
// largest magnitude and its code.  From memory, to codes and back: weights of 5120 x 27648 in
// bf16 81 and 78 us (425 MB, 5.2 and 5.4 TB/s; a copy does 4.9), of 5003 x 27001 in fp32 129
// and 125, of 2048 x 11008 in bf16 16.6 and 16.2 (68 MB: too short for that rate).
// Activations of 64 x 5120 are 2.7 us of latency, of 8192 x 5120 in bf16 27 us (126 MB).
#include "serve_internal.h"

namespace awsrc {

namespace {

typedef uint32_t u32_any __attribute__((aligned(1)));
typedef uint32_t u32x2_any __attribute__((ext_vector_type(2), aligned(1)));

// Which eight columns of a block of 128 a lane of its sixteen takes: in two groups of four where that lets neighbouring lanes
// read and write 16 bytes side by side (fp32), else all together.  `at` and `second` count from the block's first.
template <typename T>
struct Part {
  static constexpr bool kTwo = sizeof(T) == 4;
  int at;
  __device__ __forceinline__ Part(int lane) : at((lane & 15) * (kTwo ? 4 : 8)) {}
  static constexpr int second = kTwo ? 64 : 4;  // from the first four columns to the others
};

// A lane's eight values of a block at x, of whose columns n exist (the others are 0).
template <typename T>
__device__ __forceinline__ void load_part(const T* __restrict__ x, Part<T> p, int64_t n, float (&v)[8]) {
  if constexpr (Part<T>::kTwo) {
    typedef float V __attribute__((ext_vector_type(4), aligned(4)));
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int at = p.at + h * Part<T>::second;
      if (at + 4 <= n) {
        const V w = *reinterpret_cast<const V*>(x + at);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[4 * h + e] = w[e];
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[4 * h + e] = at + e < n ? x[at + e] : 0.0f;
      }
    }
  } else {
    load8_any(x + p.at, n - p.at, v);
  }
}

// The same of eight rows, all of whose loads are on their way before a value is converted.
template <typename T>
__device__ __forceinline__ void load_parts(const T* const (&x)[8], Part<T> p, int64_t n, float (&v)[8][8]) {
  constexpr int kPer = 16 / sizeof(T), kLoads = 8 / kPer;
  typedef T V __attribute__((ext_vector_type(16 / sizeof(T)), aligned(sizeof(T))));
  if (p.at + Part<T>::second + 4 <= n) {
    V w[8][kLoads];
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int h = 0; h < kLoads; ++h) w[i][h] = *reinterpret_cast<const V*>(x[i] + p.at + h * Part<T>::second);
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) v[i][e] = to_f32((T)w[i][e / kPer][e % kPer]);
  } else {
#pragma unroll
    for (int i = 0; i < 8; i += 2) {  // (two rows at a time: their addresses take registers)
      T w[2][8];
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        const int e = j & 7, at = p.at + (e < 4 ? e : Part<T>::second + e - 4);
        w[j >> 3][e] = x[i + (j >> 3)][at < n ? at : 0];
      }
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        const int e = j & 7, at = p.at + (e < 4 ? e : Part<T>::second + e - 4);
        v[i + (j >> 3)][e] = at < n ? to_f32(w[j >> 3][e]) : 0.0f;
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  }
}

// And its codes, to any byte address.
template <typename T>
__device__ __forceinline__ void store_part(uint8_t* __restrict__ c, Part<T> p, int64_t n, uint2 w) {
  if (p.at + Part<T>::second + 4 <= n) {
    if constexpr (Part<T>::kTwo) {
      *reinterpret_cast<u32_any*>(c + p.at) = w.x;
      *reinterpret_cast<u32_any*>(c + p.at + Part<T>::second) = w.y;
    } else {
      *reinterpret_cast<u32x2_any*>(c + p.at) = u32x2_any{w.x, w.y};
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int at = p.at + (e < 4 ? e : Part<T>::second + e - 4);
      if (at < n) c[at] = (uint8_t)((e < 4 ? w.x : w.y) >> (8 * (e & 3)));
    }
  }
}

// Blocks of 1 x 128: sixteen lanes a block, eight values each; a wavefront
// takes 512 columns of a row.
template <typename T>
__global__ __launch_bounds__(256) void k_quantize_blocks_row(const T* __restrict__ X, int64_t rows, int64_t cols, int64_t ldx,
                                                             uint8_t* __restrict__ codes, int64_t ldc,
                                                             float* __restrict__ scale, uint32_t strips, int64_t n_wg) {
  constexpr int R = 4;  // rows of a workgroup
  __shared__ float s_scale[4][R];
  const uint32_t wg = workgroup<256>();
  if (wg >= n_wg) return;
  const int64_t row0 = (int64_t)(wg / strips) * R, row = row0 + (threadIdx.x >> 6);
  const int64_t strip = wg % strips;
  const int lane = threadIdx.x & 63;
  const int64_t at = strip * 512 + (lane >> 4) * kBlockF8;  // the first column of this lane's block
  const Part<T> part(lane);
  float v[8], m = 0.0f;
  load_part(X + (row < rows ? row : rows - 1) * ldx + at, part, cols - at, v);
#pragma unroll
  for (int e = 0; e < 8; ++e) m = amax_keep(m, v[e]);
  const float s = scale_of_amax_f8(amax_of_16(m));
  if (row < rows) store_part(codes + row * ldc + at, part, cols - at, codes8_f8(v, inverse_scale(s), s > 0.0f));
  if ((lane & 15) == 0) s_scale[lane >> 4][threadIdx.x >> 6] = s;
  __syncthreads();
  const int64_t blocks = (cols + kBlockF8 - 1) / kBlockF8;
  for (int i = threadIdx.x; i < 4 * R; i += 256) {
    const int64_t b = strip * 4 + i / R, r = row0 + i % R;
    if (b < blocks && r < rows) scale[b * rows + r] = s_scale[i / R][i % R];
  }
}

// Blocks of 128 x 128, one a workgroup, held in registers between its largest magnitude and its codes (2048 x 11008 in bf16:
// 21.2 us where a row's values are converted before the next row is asked for).
template <typename T>
__global__ __launch_bounds__(256) void k_quantize_blocks_square(const T* __restrict__ X, int64_t rows, int64_t cols,
                                                                int64_t ldx, uint8_t* __restrict__ codes, int64_t ldc,
                                                                float* __restrict__ scale, uint32_t col_blocks, int64_t n_wg) {
  __shared__ float peak[4];
  const uint32_t wg = workgroup<256>();
  if (wg >= n_wg) return;
  const int64_t rb = wg / col_blocks, cb = wg % col_blocks;
  const int64_t row0 = rb * kBlockF8 + (threadIdx.x >> 4), at = cb * kBlockF8;
  const Part<T> part(threadIdx.x);
  const T* x[8];  // (rows past the end count the last one twice)
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = X + (row0 + 16 * i < rows ? row0 + 16 * i : rows - 1) * ldx + at;
  float v[8][8];
  load_parts(x, part, cols - at, v);
  float m = 0.0f;
#pragma unroll
  for (int i = 0; i < 8; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) m = amax_keep(m, v[i][e]);
  m = amax_of_16(m);
  m = amax_keep(m, __shfl_xor(m, 16, 64));
  m = amax_keep(m, __shfl_xor(m, 32, 64));
  if ((threadIdx.x & 63) == 0) peak[threadIdx.x >> 6] = m;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < 4; ++w) m = amax_keep(m, peak[w]);
  const float s = scale_of_amax_f8(m);
  const float inv = inverse_scale(s);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int64_t row = row0 + 16 * i;
    if (row < rows) store_part(codes + row * ldc + at, part, cols - at, codes8_f8(v[i], inv, s > 0.0f));
  }
  if (threadIdx.x == 0) scale[wg] = s;
}

// Values of codes: eight a lane, 512 columns of a row a wavefront.  Where rows do not lie on cache lines, neighbouring strips go to
// one XCD, whose L2 joins the lines that they share (5003 x 27001 into fp32 156 us, 126 so, into bf16 88 and 79; on lines
// the other way is better: 5120 x 27648 into bf16 78, 80 so).
template <typename T>
__global__ __launch_bounds__(256) void k_dequantize_blocks(const uint8_t* __restrict__ codes, int64_t ldc,
                                                           const float* __restrict__ scale, int64_t rows, int64_t cols,
                                                           bool square, T* __restrict__ out, int64_t ldo, uint32_t strips,
                                                           int64_t n_wg, bool side_by_side) {
  uint32_t wg = workgroup<256>();
  if (wg >= n_wg) return;
  if (side_by_side) wg = (uint32_t)xcd_item(wg, n_wg);
  const int64_t row = (int64_t)(wg / strips) * 4 + (threadIdx.x >> 6);
  const int64_t at = (int64_t)(wg % strips) * 512 + ((threadIdx.x & 63) >> 4) * kBlockF8;
  if (row >= rows || at >= cols) return;
  const int64_t blocks = (cols + kBlockF8 - 1) / kBlockF8, n = cols - at;
  const float s = square ? scale[row / kBlockF8 * blocks + at / kBlockF8] : scale[at / kBlockF8 * rows + row];
  const uint8_t* c = codes + row * ldc + at;
  T* o = out + row * ldo + at;
  const Part<T> part(threadIdx.x);
  if (part.at + Part<T>::second + 4 <= n) {
    uint32_t w[2];
    if constexpr (Part<T>::kTwo) {
      w[0] = *reinterpret_cast<const u32_any*>(c + part.at);
      w[1] = *reinterpret_cast<const u32_any*>(c + part.at + Part<T>::second);
    } else {
      const u32x2_any x = *reinterpret_cast<const u32x2_any*>(c + part.at);
      w[0] = x[0];
      w[1] = x[1];
    }
    float y[8];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const auto a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[i], false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[i], true);
      y[4 * i] = rounded(a[0] * s);
      y[4 * i + 1] = rounded(a[1] * s);
      y[4 * i + 2] = rounded(b[0] * s);
      y[4 * i + 3] = rounded(b[1] * s);
    }
    constexpr int kPer = 16 / sizeof(T);
    typedef T V __attribute__((ext_vector_type(16 / sizeof(T)), aligned(sizeof(T))));
#pragma unroll
    for (int i = 0; i < 8 / kPer; ++i) {
      V z;
#pragma unroll
      for (int e = 0; e < kPer; ++e) z[e] = (T)y[i * kPer + e];
      *reinterpret_cast<V*>(o + part.at + i * Part<T>::second) = z;
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int j = part.at + (e < 4 ? e : Part<T>::second + e - 4);
      if (j < n) o[j] = (T)rounded(__builtin_amdgcn_cvt_f32_fp8((int)c[j], 0) * s);
    }
  }
}

template <typename T>
hipError_t launch(const void* X, int64_t rows, int64_t cols, int64_t ldx, int block_rows, uint8_t* codes, int64_t ldc,
                  float* scale, hipStream_t st) {
  const T* x = static_cast<const T*>(X);
  if (block_rows == 1) {
    const uint32_t strips = (uint32_t)((cols + 511) / 512);
    const int64_t n = (rows + 3) / 4 * strips;
    if (n >= (int64_t)1 << 31) return hipErrorInvalidValue;
    hipLaunchKernelGGL((k_quantize_blocks_row<T>), grid_of<256>(n), dim3(256), 0, st, x, rows, cols, ldx, codes, ldc, scale,
                       strips, n);
  } else {
    const uint32_t cb = (uint32_t)((cols + kBlockF8 - 1) / kBlockF8);
    const int64_t n = (rows + kBlockF8 - 1) / kBlockF8 * cb;
    if (n >= (int64_t)1 << 31) return hipErrorInvalidValue;
    hipLaunchKernelGGL((k_quantize_blocks_square<T>), grid_of<256>(n), dim3(256), 0, st, x, rows, cols, ldx, codes, ldc, scale,
                       cb, n);
  }
  return hipGetLastError();
}

template <typename T>
hipError_t launch_back(const uint8_t* codes, int64_t ldc, const float* scale, int64_t rows, int64_t cols, int block_rows,
                       void* out, int64_t ldo, hipStream_t st) {
  const uint32_t strips = (uint32_t)((cols + 511) / 512);
  const int64_t n = (rows + 3) / 4 * strips;
  if (n >= (int64_t)1 << 31) return hipErrorInvalidValue;
  const bool on_lines = ((reinterpret_cast<uintptr_t>(out) | (uintptr_t)(ldo * sizeof(T))) & 127) == 0;
  hipLaunchKernelGGL((k_dequantize_blocks<T>), grid_of<256>(n), dim3(256), 0, st, codes, ldc, scale, rows, cols,
                     block_rows != 1, static_cast<T*>(out), ldo, strips, n, !on_lines);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_quantize_blocks(const void* X, int x_dtype, int64_t rows, int64_t cols, int64_t ldx, int block_rows,
                                  uint8_t* codes, int64_t ldc, float* scale, hipStream_t st) {
  if (x_dtype == AWSRC_DTYPE_F32) return launch<float>(X, rows, cols, ldx, block_rows, codes, ldc, scale, st);
  if (x_dtype == AWSRC_DTYPE_BF16) return launch<__bf16>(X, rows, cols, ldx, block_rows, codes, ldc, scale, st);
  return launch<_Float16>(X, rows, cols, ldx, block_rows, codes, ldc, scale, st);
}

hipError_t launch_dequantize_blocks(const uint8_t* codes, int64_t ldc, const float* scale, int64_t rows, int64_t cols,
                                    int block_rows, void* out, int out_dtype, int64_t ldo, hipStream_t st) {
  if (out_dtype == AWSRC_DTYPE_F32) return launch_back<float>(codes, ldc, scale, rows, cols, block_rows, out, ldo, st);
  if (out_dtype == AWSRC_DTYPE_BF16) return launch_back<__bf16>(codes, ldc, scale, rows, cols, block_rows, out, ldo, st);
  return launch_back<_Float16>(codes, ldc, scale, rows, cols, block_rows, out, ldo, st);
}

}  // namespace awsrc
