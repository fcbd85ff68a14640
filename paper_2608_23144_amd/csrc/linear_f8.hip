// Products of e4m3 matrices with a scale for each block of 128:
//   out[m][n] = sum_b a_scale[b][m] b_scale[n / 128][b] sum_{k in b} A[m][k] B[n][k] + bias[n].
// One v_mfma_f32_16x16x128_f8f6f4 from a zero accumulator is a block's sums of
// a 16 x 16 tile; one fma a value then adds them with their scale.
//
// That instruction adds eight adjacent products at a time at the exponent of the largest and
// cuts off what lies 2^13 below it (measured: beside a product of 2^16 one of 8 counts, one
// of 4 does not; between the eights it adds in fp32).  The results are 1.5e-5
// rms off, a tenth of fp16's own rounding and a hundredth of bf16's.  Results in fp32
// would show it: for them the codes, which fp16 holds exactly, go as fp16 through
// v_mfma_f32_16x16x32_f16, at half the rate, which adds in fp32 throughout.
//
// Matrix-core layout: an operand lane l holds row l % 16 and 32 bytes of a block
// of 128, the same ones in both operands; the result
// lane holds column l % 16 and rows 4 (l / 16) + i.  B (the weights) takes the rows'
// place and A the columns', so that a lane ends with four consecutive n of one m,
// and with one scale of A.
#include "serve_internal.h"

namespace awsrc {

namespace {

typedef int32_t i32x8 __attribute__((ext_vector_type(8)));

// Eight codes as fp16.
__device__ __forceinline__ h8 halves(int lo, int hi) {
  const auto a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((uint32_t)lo, 1.0f, false);
  const auto b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((uint32_t)lo, 1.0f, true);
  const auto c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((uint32_t)hi, 1.0f, false);
  const auto d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((uint32_t)hi, 1.0f, true);
  return h8{(_Float16)a[0], (_Float16)a[1], (_Float16)b[0], (_Float16)b[1],
            (_Float16)c[0], (_Float16)c[1], (_Float16)d[0], (_Float16)d[1]};
}

// A block's sums of a 16 x 16 tile, in fp32 throughout where FULL.
template <bool FULL>
__device__ __forceinline__ fl4 block_sums(i32x8 w, i32x8 x) {
  fl4 p = {0, 0, 0, 0};
  if constexpr (FULL) {
#pragma unroll
    for (int i = 0; i < 8; i += 2) p = __builtin_amdgcn_mfma_f32_16x16x32_f16(halves(w[i], w[i + 1]), halves(x[i], x[i + 1]), p, 0, 0, 0);
    return p;
  }
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, x, p, 0, 0, 0, 0, 0, 0);
}

// 16 bytes of which `left` belong to the sum, zeros past them.
__device__ __forceinline__ i32x4 piece(const uint8_t* p, int64_t left) {
  i32x4 w = {0, 0, 0, 0};
  if (left > 0) w = *reinterpret_cast<const i32x4*>(p);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int64_t m = left - 4 * e;
    if (m < 4) w[e] = m <= 0 ? 0 : w[e] & (int)((1u << (8 * m)) - 1u);
  }
  return w;
}

// A wavefront makes 16 x 16 values straight from memory.
template <typename TO>
__global__ __launch_bounds__(256) void k_matmul_f8(LinearF8Args a, int64_t tiles_n, int64_t tiles) {
  const int64_t tile = (int64_t)workgroup<256>() * 4 + (threadIdx.x >> 6);
  if (tile >= tiles) return;
  const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
  const int64_t m0 = tile / tiles_n * 16, n0 = tile % tiles_n * 16;
  const int64_t m = m0 + r < a.M ? m0 + r : a.M - 1;  // (rows that do not exist read the last one and are not stored)
  const uint8_t* pa = a.A + m * a.lda + 32 * g;
  const uint8_t* pb = a.B + (n0 + r < a.N ? n0 + r : a.N - 1) * a.ldb + 32 * g;
  const int64_t blocks = (a.K + kBlockF8 - 1) / kBlockF8;
  const float* sb = a.b_scale + n0 / kBlockF8 * blocks;
  fl4 acc = {0, 0, 0, 0};
  for (int64_t b = 0; b < blocks; ++b) {
    i32x8 w, x;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int64_t left = a.K - (b * kBlockF8 + 32 * g + 16 * h);
      const i32x4 u = piece(pb + b * kBlockF8 + 16 * h, left), v = piece(pa + b * kBlockF8 + 16 * h, left);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        w[4 * h + e] = u[e];
        x[4 * h + e] = v[e];
      }
    }
    const fl4 p = block_sums<sizeof(TO) == 4>(w, x);
    const float s = a.a_scale[b * a.M + m] * sb[b];
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[e] = __builtin_fmaf(p[e], s, acc[e]);
  }
  if (m0 + r >= a.M) return;
  TO* o = static_cast<TO*>(a.out) + m * a.ldo;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int64_t n = n0 + 4 * g + e;
    if (n < a.N) o[n] = (TO)rounded(acc[e] + (a.bias ? a.bias[n] : 0.0f));
  }
}

template <typename TO>
hipError_t launch(const LinearF8Args& a, hipStream_t st) {
  const int64_t tn = (a.N + 15) / 16, tiles = (a.M + 15) / 16 * tn;
  if (tiles >= (int64_t)1 << 32) return hipErrorInvalidValue;
  hipLaunchKernelGGL((k_matmul_f8<TO>), grid_of<256>((tiles + 3) / 4), dim3(256), 0, st, a, tn, tiles);
  return hipGetLastError();
}

}  // namespace

size_t matmul_f8_ws_bytes(int64_t, int64_t, int64_t) { return 0; }

hipError_t launch_matmul_f8(const LinearF8Args& a, void*, hipStream_t st) {
  if (a.out_dtype == AWSRC_DTYPE_F32) return launch<float>(a, st);
  if (a.out_dtype == AWSRC_DTYPE_BF16) return launch<__bf16>(a, st);
  return launch<_Float16>(a, st);
}

}  // namespace awsrc
