// Internal declarations of the 8-bit serving operators (quant_i8.hip,
// linear_i8.hip, kv_cache.hip, kv_attention.hip; not part of the ABI).
#pragma once

#include "awsrc_internal.h"

namespace awsrc {

typedef int32_t i32x4 __attribute__((ext_vector_type(4)));
typedef int32_t i32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef float fl4 __attribute__((ext_vector_type(4)));
typedef float fl16 __attribute__((ext_vector_type(16)));
typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));

// A row or block whose largest magnitude lies below this is stored as zeros
// with scale 0, so that scales and their inverses stay normal numbers.
constexpr float kTinyAmax = 0x1p-100f;

// Integer sums of int8 products stay below 2^31 up to this length, -128 included.
constexpr int64_t kMaxSumI8 = 131071;

// The 8-bit recipe (fp32, each operation rounded once): the scale of a
// largest magnitude, NaN where that is not finite.
__device__ __forceinline__ float scale_of_amax(float amax) {
  if (!(amax < __builtin_inff())) return __builtin_nanf("");
  return amax < kTinyAmax ? 0.0f : amax / 127.0f;
}
// 1 / scale, 0 for a zero scale (NaN stays NaN).
__device__ __forceinline__ float inverse_scale(float s) { return s == 0.0f ? 0.0f : 1.0f / s; }
// rint(x * inv) as a code; 0 where the product is NaN.
__device__ __forceinline__ int code_of(float x, float inv) {
  const float r = rintf(x * inv);
  return (int)fminf(fmaxf(r == r ? r : 0.0f, -127.0f), 127.0f);
}

// max of |x| that keeps a NaN (fmaxf would drop it).
__device__ __forceinline__ float amax_keep(float m, float x) {
  const float a = fabsf(x);
  return (a > m || a != a) ? a : m;
}

template <typename T>
__device__ __forceinline__ float to_f32(T x) { return (float)x; }

// Eight adjacent values on 16 bytes, as vector accesses (copies of a struct of
// eight are taken apart by the compiler and merged with the element-wise path).
template <typename T>
__device__ __forceinline__ void load_vec8(const T* __restrict__ x, float (&v)[8]) {
  if constexpr (sizeof(T) == 4) {
    const fl4 a = reinterpret_cast<const fl4*>(x)[0], b = reinterpret_cast<const fl4*>(x)[1];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = e < 4 ? a[e & 3] : b[e & 3];
  } else {
    typedef T t8 __attribute__((ext_vector_type(8)));
    const t8 w = *reinterpret_cast<const t8*>(x);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = to_f32((T)w[e]);
  }
}
template <typename T>
__device__ __forceinline__ void store_vec8(T* __restrict__ x, const float (&v)[8]) {
  if constexpr (sizeof(T) == 4) {
    reinterpret_cast<fl4*>(x)[0] = fl4{v[0], v[1], v[2], v[3]};
    reinterpret_cast<fl4*>(x)[1] = fl4{v[4], v[5], v[6], v[7]};
  } else {
    typedef T t8 __attribute__((ext_vector_type(8)));
    t8 w;
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e] = (T)v[e];
    *reinterpret_cast<t8*>(x) = w;
  }
}

// Eight values from x, of which n exist (the others are 0).
template <typename T>
__device__ __forceinline__ void load8(const T* __restrict__ x, int64_t n, bool wide, float (&v)[8]) {
  if (wide && n >= 8) {
    load_vec8(x, v);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = e < n ? to_f32(x[e]) : 0.0f;
  }
}

// Codes of eight values; `live` is false for a row whose scale is NaN.  No
// clamp: |x| <= amax gives |x inv| <= 127 (1 + 2^-22).
__device__ __forceinline__ uint2 codes8(const float (&v)[8], float inv, bool live) {
  uint32_t q[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) q[e] = live ? (uint32_t)(int)rintf(v[e] * inv) : 0u;
  uint2 o;
  o.x = (q[0] & 255) | (q[1] & 255) << 8 | (q[2] & 255) << 16 | q[3] << 24;
  o.y = (q[4] & 255) | (q[5] & 255) << 8 | (q[6] & 255) << 16 | q[7] << 24;
  return o;
}

// A grid of n < 2^31 workgroups.  A launch counts its threads along x in 32 bits, and the runtime lets more of them wrap
// around without an error (16.8 M workgroups of 256 ran 65,536): past 2^31 threads they go along y, in rows of 2^31
// threads.  workgroup() is a workgroup's number, in the last row n or more.
template <int THREADS>
dim3 grid_of(int64_t n) {
  constexpr int64_t kRow = ((int64_t)1 << 31) / THREADS;
  return n <= kRow ? dim3((unsigned)n) : dim3((unsigned)kRow, (unsigned)((n + kRow - 1) / kRow));
}
template <int THREADS>
__device__ __forceinline__ uint32_t workgroup() {
  return blockIdx.x + blockIdx.y * (uint32_t)(((int64_t)1 << 31) / THREADS);
}

struct LinearArgs {
  const int8_t* A;       // [M][lda] activation codes
  int64_t lda;
  const float* a_scale;  // [M]
  const int8_t* B;       // [N][ldb] weight codes
  int64_t ldb;
  const float* b_scale;  // [N]
  const float* bias;     // [N] or NULL
  int64_t M, N, K;
  void* out;             // [M][ldo]
  int out_dtype;
  int64_t ldo;
};

hipError_t launch_quantize_rows(const void* X, int x_dtype, int64_t rows, int64_t cols, int64_t ldx, int8_t* codes,
                                int64_t ldc, float* scale, hipStream_t st);
size_t matmul_i8_ws_bytes(int64_t M, int64_t N, int64_t K);
hipError_t launch_matmul_i8(const LinearArgs& a, void* ws, hipStream_t st);
// Whether a linear layer of this shape quantizes its rows in the product's kernel, and that kernel (a.A unused).
bool linear_i8_fused(int64_t M, int64_t N, int64_t K);
hipError_t launch_linear_i8_fused(const LinearArgs& a, const void* X, int x_dtype, int64_t ldx, hipStream_t st);

struct AppendArgs {
  awsrc_kv_cache c;
  const void *k, *v, *q;   // q may be NULL
  int64_t ldk, ldv, ldq, ldqo;
  int dtype, q_heads;
  void* q_out;
  const float *cos, *sin;  // [rope_len][rot / 2]
  int64_t rope_len;
  int rot, interleaved;
  int n_seq;
  int64_t n_rows;
  const int32_t *cu, *kv_len, *table;
  int64_t table_ld;
  int64_t max_new;
};
hipError_t launch_kv_append(const AppendArgs& a, hipStream_t st);

struct ReadArgs {
  awsrc_kv_cache c;
  int n_seq;
  int64_t n_rows;
  const int32_t *cu, *kv_len, *table;
  int64_t table_ld;
  int64_t max_rows;
  void *k_out, *v_out;
  int dtype;
};
hipError_t launch_kv_read(const ReadArgs& a, hipStream_t st);

struct AttentionArgs {
  awsrc_kv_cache c;
  const void* q;
  int64_t ldq;
  int dtype, q_heads;
  int n_seq;
  int64_t n_rows;
  const int32_t *cu, *kv_len, *table;
  int64_t table_ld;
  int64_t max_new, max_kv;
  float scale;
  int causal;
  void* out;
  int64_t ldo;
};
size_t kv_attention_ws_bytes(const AttentionArgs& a);
hipError_t launch_kv_attention(const AttentionArgs& a, void* ws, hipStream_t st);

}  // namespace awsrc
