// Internal declarations of the serving operators (quant_i8.hip, linear_i8.hip,
// quant_f8.hip, linear_f8.hip, kv_cache.hip, kv_attention.hip, kv_plan.hip,
// verify.hip; not part of the ABI).
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

// max of |x| that keeps a NaN (fmaxf would drop it); two values an instruction.  With a comparison and a choice in its place
// the int8 layer of 1 x 2560 x 2048 takes 4.8 us, 4.4 so, 48 appended tokens 10.5 and 10.1, long attention 30.3 and 29.4.
__device__ __forceinline__ float amax_keep(float m, float x) { return __builtin_elementwise_maximum(m, fabsf(x)); }

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

// A value that is fp32 before it is rounded to its type.  Without it the compiler takes an operation and the conversion to
// fp16 after it as one instruction, which does not round in between, in some places and not in others.
__device__ __forceinline__ float rounded(float y) {
  asm("" : "+v"(y));
  return y;
}

// Four values of a result row, those of them that exist.
template <typename TO>
__device__ __forceinline__ void store4(TO* o, const float (&y)[4], int64_t n, int64_t N, bool wide) {
  if (wide && n + 3 < N) {
    struct alignas(4 * sizeof(TO)) V { TO v[4]; } w;
#pragma unroll
    for (int i = 0; i < 4; ++i) w.v[i] = (TO)y[i];
    *reinterpret_cast<V*>(o + n) = w;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (n + i < N) o[n + i] = (TO)y[i];
  }
}

// Lane j of a quad of neighbouring lanes gets as v[i] what lane i of it loaded as v[j].
__device__ __forceinline__ void turn_quads(i32x4 (&v)[4], int lane) {
  const bool odd = lane & 1, high = lane & 2;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    int x[4], y[4];
#pragma unroll
    for (int i = 0; i < 4; i += 2) {
      const int p = __builtin_amdgcn_mov_dpp(v[i + 1][e], 0xB1, 0xF, 0xF, true);  // of lane ^ 1
      const int q = __builtin_amdgcn_mov_dpp(v[i][e], 0xB1, 0xF, 0xF, true);
      x[i] = odd ? p : v[i][e];
      x[i + 1] = odd ? v[i + 1][e] : q;
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int p = __builtin_amdgcn_mov_dpp(x[i + 2], 0x4E, 0xF, 0xF, true);  // of lane ^ 2
      const int q = __builtin_amdgcn_mov_dpp(x[i], 0x4E, 0xF, 0xF, true);
      y[i] = high ? p : x[i];
      y[i + 2] = high ? x[i + 2] : q;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i][e] = y[i];
  }
}

// A barrier for LDS contents alone: __syncthreads() would also wait for every
// fill that is still to come.
__device__ __forceinline__ void sync_lds() {
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

// Columns of a block of e4m3 codes with one scale, and rows of a weight block.
constexpr int kBlockF8 = 128;

// The e4m3 recipe's scale of a block's largest magnitude, NaN where that is not finite.
__device__ __forceinline__ float scale_of_amax_f8(float amax) {
  if (!(amax < __builtin_inff())) return __builtin_nanf("");
  return amax < kTinyAmax ? 0.0f : amax / 448.0f;
}

// e4m3 codes of eight values; `live` is false for a block whose scale is 0 or NaN.  No clamp: |x| <= amax gives
// |x inv| <= 448 (1 + 2^-22), which rounds to 448 (the next border is 464).
__device__ __forceinline__ uint2 codes8_f8(const float (&v)[8], float inv, bool live) {
  uint32_t w[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    int x = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * i] * inv, v[4 * i + 1] * inv, 0, false);
    x = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * i + 2] * inv, v[4 * i + 3] * inv, x, true);
    w[i] = live ? (uint32_t)x : 0u;
  }
  uint2 o;
  o.x = w[0];
  o.y = w[1];
  return o;
}

// The largest of amax over the 16 lanes of a row of lanes (NaN where one has it).
__device__ __forceinline__ float amax_of_16(float m) {
#define AWSRC_ROR(n) m = amax_keep(m, __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, m), 0x120 + n, 0xF, 0xF, true)))
  AWSRC_ROR(8);
  AWSRC_ROR(4);
  AWSRC_ROR(2);
  AWSRC_ROR(1);
#undef AWSRC_ROR
  return m;
}

// Inclusive sums over a wavefront's lanes, or (ROW) over each 16 of them, of 64-bit values; by moves between lanes' registers.
template <int CTRL, int ROWS, typename T>
__device__ __forceinline__ T add_from(T x) {
  static_assert(sizeof(T) == 8, "64-bit values");
  const uint64_t b = __builtin_bit_cast(uint64_t, x);
  const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)b, CTRL, ROWS, 0xF, false);
  const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)(b >> 32), CTRL, ROWS, 0xF, false);
  return x + __builtin_bit_cast(T, (uint64_t)hi << 32 | lo);
}
template <typename T>
__device__ __forceinline__ T scan_row(T x) {
  x = add_from<0x111, 0xF>(x);  // from the lanes 1, 2, 4 and 8 before, in each row of 16
  x = add_from<0x112, 0xF>(x);
  x = add_from<0x114, 0xF>(x);
  return add_from<0x118, 0xF>(x);
}
template <typename T>
__device__ __forceinline__ T scan_wave(T x) {
  x = add_from<0x142, 0xA>(scan_row(x));  // the last lane of the row before, into rows 1 and 3
  return add_from<0x143, 0xC>(x);         // lane 31 into rows 2 and 3
}
template <typename T>
__device__ __forceinline__ T of_lane(T x, int lane) {
  const uint64_t b = __builtin_bit_cast(uint64_t, x);
  const uint32_t lo = __builtin_amdgcn_readlane((int)(uint32_t)b, lane), hi = __builtin_amdgcn_readlane((int)(uint32_t)(b >> 32), lane);
  return __builtin_bit_cast(T, (uint64_t)hi << 32 | lo);
}
// Inclusive sums of N values over the threads of a workgroup of 4, 8 or 16 wavefronts (W), in their order; `total` is everyone's.
// Every thread of the workgroup calls it; sums may be written again after the workgroup's next barrier.
template <int W, int N, typename T>
__device__ __forceinline__ void scan_workgroup(T (&x)[N], T (&total)[N], T (*sums)[W]) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
  for (int i = 0; i < N; ++i) x[i] = scan_wave(x[i]);
  if (lane == 63)
#pragma unroll
    for (int i = 0; i < N; ++i) sums[i][wave] = x[i];
  __syncthreads();
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const T upto = scan_row((lane & 15) < W ? sums[i][lane & 15 & (W - 1)] : T(0));
    total[i] = of_lane(upto, W - 1);
    if (wave) x[i] += of_lane(upto, wave - 1);
  }
}

// Eight values from x at any alignment (memory takes vectors at any byte), of which n exist (the others are 0).
template <typename T>
__device__ __forceinline__ void load8_any(const T* __restrict__ x, int64_t n, float (&v)[8]) {
  if (n >= 8) {
    typedef T V __attribute__((ext_vector_type(16 / sizeof(T)), aligned(sizeof(T))));
    constexpr int kPer = 16 / sizeof(T);
#pragma unroll
    for (int i = 0; i < 8 / kPer; ++i) {
      const V w = *reinterpret_cast<const V*>(x + i * kPer);
#pragma unroll
      for (int e = 0; e < kPer; ++e) v[i * kPer + e] = to_f32((T)w[e]);
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = e < n ? to_f32(x[e]) : 0.0f;
  }
}

struct LinearF8Args {
  const uint8_t* A;      // [M][lda] activation codes
  int64_t lda;
  const float* a_scale;  // [ceil(K / 128)][M]
  const uint8_t* B;      // [N][ldb] weight codes
  int64_t ldb;
  const float* b_scale;  // [ceil(N / 128)][ceil(K / 128)]
  const float* bias;     // [N] or NULL
  int64_t M, N, K;
  void* out;             // [M][ldo]
  int out_dtype;
  int64_t ldo;
};

hipError_t launch_quantize_blocks(const void* X, int x_dtype, int64_t rows, int64_t cols, int64_t ldx, int block_rows,
                                  uint8_t* codes, int64_t ldc, float* scale, hipStream_t st);
hipError_t launch_dequantize_blocks(const uint8_t* codes, int64_t ldc, const float* scale, int64_t rows, int64_t cols,
                                    int block_rows, void* out, int out_dtype, int64_t ldo, hipStream_t st);
size_t matmul_f8_ws_bytes(int64_t M, int64_t N, int64_t K);
hipError_t launch_matmul_f8(const LinearF8Args& a, void* ws, hipStream_t st);
// Whether a linear layer of this shape quantizes its rows in the product's kernel, and that kernel (a.A unused).
bool linear_f8_fused(int64_t M, int64_t N, int64_t K);
hipError_t launch_linear_f8_fused(const LinearF8Args& a, const void* X, int x_dtype, int64_t ldx, hipStream_t st);

struct PlanArgs {
  awsrc_page_pool pool;
  int n_seq;
  const int32_t *kv_len, *keep, *new_len;
  int32_t* table;
  int64_t table_ld, max_rows;
  int32_t *kv_out, *n_free_out, *cu, *row_seq, *row_pos;
  int64_t* row_slot;
};
size_t kv_plan_ws_bytes(int n_seq, int64_t max_rows);
hipError_t launch_kv_plan(const PlanArgs& a, void* ws, hipStream_t st);

struct VerifyArgs {
  const void *p, *q;  // q may be NULL
  int64_t ldp, ldq;
  int dtype;
  int64_t vocab;
  int n_seq;
  int64_t n_rows;
  const int32_t *cu, *tokens;
  const float* u;
  const int32_t* kv_len;  // NULL where keep is
  int32_t *tokens_out, *n_out, *keep;
};
size_t verify_ws_bytes(int n_seq, int64_t vocab);
hipError_t launch_verify(const VerifyArgs& a, void* ws, hipStream_t st);

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
