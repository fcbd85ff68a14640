// Products of int8 matrices with one scale per row of each operand:
//   out[m][n] = a_scale[m] b_scale[n] sum_k A[m][k] B[n][k] + bias[n],
// the sum exact in int32 on v_mfma_i32_16x16x64_i8, the epilogue in fp32 with
// one rounding to the output type.
//
// Matrix-core layout: an operand lane l holds row l % 16 and the 16 bytes
// [16 (l / 16), + 16) of a 64-byte step; the result lane holds column l % 16
// and rows 4 (l / 16) + i.  B (the weights) takes the rows' place and A the
// columns', so that a lane ends with four consecutive n of one m.
#include "serve_internal.h"

namespace awsrc {

namespace {

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

// 16 bytes of an operand row at byte k, zero past K (rows are readable to the
// next multiple of 16) and for rows that do not exist.
__device__ __forceinline__ i32x4 load_chunk(const int8_t* __restrict__ p, int64_t ld, int64_t row, int64_t rows,
                                            int64_t k, int64_t K) {
  i32x4 v = {0, 0, 0, 0};
  if (row < rows && k < K) {
    v = *reinterpret_cast<const i32x4*>(p + row * ld + k);
    if (k + 16 > K) {
      const int left = (int)(K - k);
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const int b = left - 4 * w;
        v[w] = b <= 0 ? 0 : b >= 4 ? v[w] : (v[w] & (int)((1u << (8 * b)) - 1u));
      }
    }
  }
  return v;
}

// One workgroup: 16 output columns and 16 rows, the sum split over 4 wavefronts.
template <typename TO>
__global__ __launch_bounds__(256) void k_matmul_i8_rows(LinearArgs a) {
  __shared__ i32x4 part[4][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t n0 = (int64_t)blockIdx.x * 16, m0 = (int64_t)blockIdx.y * 16;
  const int r = lane & 15, g = lane >> 4;
  i32x4 acc = {0, 0, 0, 0};
  for (int64_t k = (int64_t)wave * 64; k < a.K; k += 256) {
    const i32x4 w = load_chunk(a.B, a.ldb, n0 + r, a.N, k + 16 * g, a.K);
    const i32x4 x = load_chunk(a.A, a.lda, m0 + r, a.M, k + 16 * g, a.K);
    acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(w, x, acc, 0, 0, 0);
  }
  part[wave][lane] = acc;
  __syncthreads();
  if (wave) return;
#pragma unroll
  for (int w = 1; w < 4; ++w) acc += part[w][lane];
  const int64_t m = m0 + r, n = n0 + 4 * g;
  if (m >= a.M) return;
  const float sa = a.a_scale[m];
  float y[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int64_t nn = n + i < a.N ? n + i : a.N - 1;
    y[i] = (float)acc[i] * (sa * a.b_scale[nn]);
    if (a.bias) y[i] += a.bias[nn];
  }
  TO* o = static_cast<TO*>(a.out) + m * a.ldo;
  store4(o, y, n, a.N, ((reinterpret_cast<uintptr_t>(a.out) | (uintptr_t)(a.ldo * sizeof(TO))) & (4 * sizeof(TO) - 1)) == 0);
}

template <typename TO>
hipError_t launch(const LinearArgs& a, hipStream_t st) {
  hipLaunchKernelGGL((k_matmul_i8_rows<TO>), dim3((unsigned)((a.N + 15) / 16), (unsigned)((a.M + 15) / 16)), dim3(256),
                     0, st, a);
  return hipGetLastError();
}

}  // namespace

size_t matmul_i8_ws_bytes(int64_t, int64_t, int64_t) { return 0; }

hipError_t launch_matmul_i8(const LinearArgs& a, void*, hipStream_t st) {
  if (a.out_dtype == AWSRC_DTYPE_F32) return launch<float>(a, st);
  if (a.out_dtype == AWSRC_DTYPE_BF16) return launch<__bf16>(a, st);
  return launch<_Float16>(a, st);
}

}  // namespace awsrc
