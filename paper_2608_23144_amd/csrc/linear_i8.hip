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

// Tiles through LDS, for products with enough rows to fill the matrix cores.
//
// A workgroup makes BM rows (m) times BN columns (n) of the result, a
// wavefront WM x WN of them as 32 x 32 tiles of v_mfma_i32_32x32x32_i8.  The sum
// advances 128 bytes at a time through two LDS stages filled by direct
// global-to-LDS loads, which leave the registers to the sums.  A stage's rows
// of 128 bytes are 8 pieces of 16; piece p of row r lies at place p ^ key(r), with
// keys that differ over any 8 lanes that read together, so that neither the
// fragment reads nor the fills collide in banks.  The fills of step t + 1 and the
// fragment reads of the next 32 bytes are issued before the products of the
// current ones.
//
// Rows and pieces past the operands' ends come from beyond the buffer resource
// and arrive as zeros.  Where K is no multiple of 16 the bytes past it are
// cleared in LDS, on A's side alone (0 times whatever B holds).
//
// Weight row 8 b + 4 h + i of a 32-row tile carries column 16 h + 4 b + i, so
// that a lane (half h) ends with 16 consecutive columns of one result row.
constexpr int kStep = 128;

__device__ __forceinline__ int key_a(int row) { return row & 7; }
__device__ __forceinline__ int key_b(int row) { return (row & 3) | ((row >> 2) & 4); }

template <int BM, int BN, int WM, int WN>
struct TileShape {
  static constexpr int kWaves = (BM / WM) * (BN / WN);
  static constexpr int kThreads = 64 * kWaves;
  static constexpr int kStage = (BM + BN) * kStep;
};

template <int BM, int BN, int WM, int WN, int OCC, typename TO>
__global__ __launch_bounds__((TileShape<BM, BN, WM, WN>::kThreads), OCC) void k_matmul_i8_tile(LinearArgs a, int tiles_m,
                                                                                               int tiles_n) {
  using S = TileShape<BM, BN, WM, WN>;
  constexpr int TM = WM / 32, TN = WN / 32;
  constexpr int NA = BM * 8 / S::kThreads, NB = BN * 8 / S::kThreads;  // 16-byte pieces per thread and step
  constexpr int kRows = S::kThreads / 8;                              // rows that one round of fills covers
  extern __shared__ __attribute__((aligned(1024))) char lds[];

  // neighbouring tiles on one XCD, in bands of 8 tile rows, share operands in its L2
  const int total = tiles_m * tiles_n;
  const int id = (int)xcd_item(blockIdx.x, total);
  const int band = id / (8 * tiles_n), in = id - band * 8 * tiles_n;
  const int bm = tiles_m - band * 8 < 8 ? tiles_m - band * 8 : 8;
  const int64_t m0 = (int64_t)(band * 8 + in % bm) * BM, n0 = (int64_t)(in / bm) * BN;

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = (wave % (BM / WM)) * WM, wn = (wave / (BM / WM)) * WN;
  const int K = (int)a.K, K16 = (K + 15) & ~15;

  // buffer resources from the tile's first rows to the operands' last readable bytes
  const int64_t ma = a.M - m0, nb = a.N - n0;
  const int64_t end_a = (ma - 1) * a.lda + K16, end_b = (nb - 1) * a.ldb + K16;
  const __amdgpu_buffer_rsrc_t ra = __builtin_amdgcn_make_buffer_rsrc(
      const_cast<int8_t*>(a.A + m0 * a.lda), 0, (int)(end_a < 0x7FFFFFFF ? end_a : 0x7FFFFFFF), 0x00020000);
  const __amdgpu_buffer_rsrc_t rb = __builtin_amdgcn_make_buffer_rsrc(
      const_cast<int8_t*>(a.B + n0 * a.ldb), 0, (int)(end_b < 0x7FFFFFFF ? end_b : 0x7FFFFFFF), 0x00020000);

  // fills: thread -> LDS row tid / 8 (+ kRows per round), place tid % 8
  const int frow = tid >> 3;
  const int pa = ((tid & 7) ^ key_a(frow)) * 16, pb = ((tid & 7) ^ key_b(frow)) * 16;
  const uint32_t oa = (uint32_t)frow * (uint32_t)a.lda + pa, ob = (uint32_t)frow * (uint32_t)a.ldb + pb;
  const uint32_t sa = kRows * (uint32_t)a.lda, sb = kRows * (uint32_t)a.ldb;
  typedef __attribute__((address_space(3))) void* lds_ptr;
  auto fill = [&](int stage, int k) {
    char* base = lds + stage * S::kStage + wave * 1024;
    const bool ina = k + pa < K, inb = k + pb < K;
#pragma unroll
    for (int i = 0; i < NA; ++i)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(ra, (lds_ptr)(base + i * kRows * kStep), 16,
                                               ina ? (int)(oa + i * sa + k) : (int)0x80000000, 0, 0, 0);
#pragma unroll
    for (int i = 0; i < NB; ++i)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rb, (lds_ptr)(base + (BM + i * kRows) * kStep), 16,
                                               inb ? (int)(ob + i * sb + k) : (int)0x80000000, 0, 0, 0);
  };
  // fragments: lane -> row lane % 32 of the tile, 16-byte piece 2 ks + lane / 32
  const int half = lane >> 5, r = lane & 31;
  const int rb_n = ((r >> 2) & 1) * 16 + (r >> 3) * 4 + (r & 3);
  const int la = (wm + r) * kStep, lb = (BM + wn + rb_n) * kStep;
  const int xa = key_a(r), xb = key_b(rb_n);
  auto frags = [&](int stage, int ks, i32x4 (&fa)[TM], i32x4 (&fb)[TN]) {
    const char* base = lds + stage * S::kStage;
    const int qa = ((2 * ks + half) ^ xa) * 16, qb = ((2 * ks + half) ^ xb) * 16;
#pragma unroll
    for (int t = 0; t < TN; ++t) fb[t] = *reinterpret_cast<const i32x4*>(base + lb + t * 32 * kStep + qb);
#pragma unroll
    for (int t = 0; t < TM; ++t) fa[t] = *reinterpret_cast<const i32x4*>(base + la + t * 32 * kStep + qa);
  };

  i32x16 acc[TN][TM];
#pragma unroll
  for (int i = 0; i < TN; ++i)
#pragma unroll
    for (int j = 0; j < TM; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0;
  auto products = [&](const i32x4 (&fa)[TM], const i32x4 (&fb)[TN]) {
#pragma unroll
    for (int i = 0; i < TN; ++i)
#pragma unroll
      for (int j = 0; j < TM; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(fb[i], fa[j], acc[i][j], 0, 0, 0);
  };

  const int steps = (K + kStep - 1) / kStep;
  // waits for this wavefront's fills, then for everyone's; clears what lies past K in A's rows of the last step
  auto arrived = [&](int stage, int t) {
    __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0)
    __syncthreads();                     // (with lgkmcnt(0): every fragment of the stage that is refilled next is read)
    if (t == steps - 1 && K != K16) {
      const int k = K - (K16 - 16), p = (K16 - 16 - t * kStep) >> 4;
      for (int row = tid; row < BM; row += S::kThreads) {
        char* c = lds + stage * S::kStage + row * kStep + (p ^ key_a(row)) * 16;
        for (int e = k; e < 16; ++e) c[e] = 0;
      }
      __syncthreads();
    }
  };

  i32x4 fa[2][TM], fb[2][TN];
  fill(0, 0);
  arrived(0, 0);
  if (steps > 1) fill(1, kStep);
  frags(0, 0, fa[0], fb[0]);
  for (int t = 0; t < steps; ++t) {
    const int st = t & 1;
#pragma unroll
    for (int ks = 0; ks < 3; ++ks) {
      frags(st, ks + 1, fa[(ks + 1) & 1], fb[(ks + 1) & 1]);
      products(fa[ks & 1], fb[ks & 1]);
    }
    if (t + 1 < steps) {
      arrived(st ^ 1, t + 1);
      if (t + 2 < steps) fill(st, (t + 2) * kStep);
      frags(st ^ 1, 0, fa[0], fb[0]);
    }
    products(fa[1], fb[1]);
  }

  // results: lane -> row wm + 32 j + r, columns wn + 32 i + 16 half + e
  const bool wide = ((reinterpret_cast<uintptr_t>(a.out) | (uintptr_t)(a.ldo * sizeof(TO))) & 15) == 0;
#pragma unroll
  for (int i = 0; i < TN; ++i) {
    const int64_t n = n0 + wn + 32 * i + 16 * half;
    float sbv[16], bias[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const int64_t nn = n + e < a.N ? n + e : a.N - 1;
      sbv[e] = a.b_scale[nn];
      bias[e] = a.bias ? a.bias[nn] : 0.0f;
    }
#pragma unroll
    for (int j = 0; j < TM; ++j) {
      const int64_t m = m0 + wm + 32 * j + r;
      if (m >= a.M) continue;
      const float sav = a.a_scale[m];
      TO* o = static_cast<TO*>(a.out) + m * a.ldo + n;
      float y[16];
#pragma unroll
      for (int e = 0; e < 16; ++e) y[e] = (float)acc[i][j][e] * (sav * sbv[e]) + bias[e];
      if (wide && n + 16 <= a.N) {
        constexpr int V = 16 / sizeof(TO);
        struct alignas(16) Piece { TO v[V]; };
#pragma unroll
        for (int p = 0; p < 16 / V; ++p) {
          Piece w;
#pragma unroll
          for (int e = 0; e < V; ++e) w.v[e] = (TO)y[p * V + e];
          *reinterpret_cast<Piece*>(o + p * V) = w;
        }
      } else {
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (n + e < a.N) o[e] = (TO)y[e];
      }
    }
  }
}

template <int BM, int BN, int WM, int WN, int OCC, typename TO>
hipError_t launch_tile(const LinearArgs& a, hipStream_t st) {
  using S = TileShape<BM, BN, WM, WN>;
  const auto k = k_matmul_i8_tile<BM, BN, WM, WN, OCC, TO>;
  const size_t lds = 2 * S::kStage;
  if (lds > 65536) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(k), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return e;
  }
  const int64_t tm = (a.M + BM - 1) / BM, tn = (a.N + BN - 1) / BN;
  if (tm * tn > 0x7FFFFFFF / 8) return hipErrorInvalidValue;
  hipLaunchKernelGGL(k, dim3((unsigned)(tm * tn)), dim3(S::kThreads), lds, st, a, (int)tm, (int)tn);
  return hipGetLastError();
}

template <typename TO>
hipError_t launch(const LinearArgs& a, hipStream_t st) {
  const int64_t t256 = ((a.M + 255) / 256) * ((a.N + 255) / 256), t128 = ((a.M + 127) / 128) * ((a.N + 127) / 128);
  if (a.M > 64) {
    if (t256 >= 192) return launch_tile<256, 256, 128, 128, 1, TO>(a, st);
    if (t128 >= 192) return launch_tile<128, 128, 64, 64, 2, TO>(a, st);
    return launch_tile<64, 64, 32, 32, 4, TO>(a, st);
  }
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
