// Products of int8 matrices with one scale per row of each operand:
//   out[m][n] = a_scale[m] b_scale[n] sum_k A[m][k] B[n][k] + bias[n],
// the sum exact in int32 on v_mfma_i32_16x16x64_i8, the epilogue in fp32 with
// one rounding to the output type.
//
// Matrix-core layout: an operand lane l holds row l % 16 and the 16 bytes
// [16 (l / 16), + 16) of a 64-byte step; the result lane holds column l % 16
// and rows 4 (l / 16) + i.  B (the weights) takes the rows' place and A the
// columns', so that a lane ends with four consecutive n of one m.
#include <type_traits>
#include "serve_internal.h"

namespace awsrc {

namespace {

// The epilogue, the same in every kernel: two roundings after the sum's own.  The asm keeps the compiler from taking the fma
// and the conversion to fp16 after it as one instruction, which does not round to fp32 in between: it did so in some of the
// kernels, where one output in 60,000 had another last bit.
__device__ __forceinline__ float scaled(int sum, float sa, float sb, float bias) {
  float y = __builtin_fmaf((float)sum, sa * sb, bias);
  asm("" : "+v"(y));
  return y;
}

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

// Up to 16 rows (or 32: R groups of 16): the weights' bytes are all that counts.  A workgroup takes 16
// weight rows (columns of the result) against all activation rows, its W
// wavefronts sharing the sum; the weights come straight from memory, four steps
// of 64 bytes ahead of the products, and the wavefronts' sums meet in LDS.
//
// The matrix cores want neighbouring lanes to hold neighbouring rows, but a CU's
// cache takes in a quad of lanes a cycle only where they read 64 bytes side by
// side.  So lane j of a quad loads piece j of its quad's four rows, and the quad
// trades them: the lane ends with 64 bytes of its own row, which are its pieces of
// four steps (13 x 2048 x 11008, weights in the last cache: 7.7 us, 11.2 with each lane loading its own;
// neither 16 wavefronts nor 8 columns a workgroup are faster: 7.6 and 7.8).
template <int W, int R, bool AHEAD>
struct RowSums {
  static constexpr int U = 4;
  const int8_t* pb[U];  // rows 4 (row / 4) + u of the weights, this lane's piece of a round
  const int8_t* pa[R][U];  // the same of R groups of 16 rows of activation codes (AHEAD: in memory, fetched with the weights)
  const int8_t *rb, *ra[R];  // this lane's own rows
  int K, wave, lane, g;
  i32x4 acc[R];
  i32x4 fb[2][U], fa[2][R][U];

  // rows that do not exist read the last one: their sums are not stored
  __device__ __forceinline__ RowSums(const LinearArgs& a, int64_t n0, int ln, int wv, const int8_t* A, int64_t lda)
      : K((int)a.K), wave(wv), lane(ln), g(ln >> 4) {
    const auto weights = [&](int r) { return a.B + (n0 + r < a.N ? n0 + r : a.N - 1) * a.ldb; };
    const auto codes = [&](int r) { return A + (r < a.M ? r : a.M - 1) * lda; };
#pragma unroll
    for (int u = 0; u < U; ++u) {
      pb[u] = weights((ln & 12) + u) + 64 * g + 16 * (ln & 3);
#pragma unroll
      for (int j = 0; j < R; ++j) pa[j][u] = codes(16 * j + (ln & 12) + u) + 64 * g + 16 * (ln & 3);
    }
    rb = weights(ln & 15);
#pragma unroll
    for (int j = 0; j < R; ++j) {
      ra[j] = codes(16 * j + (ln & 15));
      acc[j] = i32x4{0, 0, 0, 0};
    }
  }
  __device__ __forceinline__ void load(int buf, int k) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      fb[buf][u] = *reinterpret_cast<const i32x4*>(pb[u] + k);
      if constexpr (AHEAD)
#pragma unroll
        for (int j = 0; j < R; ++j) fa[buf][j][u] = *reinterpret_cast<const i32x4*>(pa[j][u] + k);
    }
  }
  __device__ __forceinline__ int rounds() const { return K / (64 * U); }
  __device__ __forceinline__ void begin() {
    if (wave < rounds()) load(0, wave * 64 * U);
  }
  __device__ __forceinline__ void products(int buf, int k) {
    turn_quads(fb[buf], lane);
#pragma unroll
    for (int j = 0; j < R; ++j) {
      if constexpr (AHEAD) turn_quads(fa[buf][j], lane);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const i32x4 x = AHEAD ? fa[buf][j][u] : *reinterpret_cast<const i32x4*>(ra[j] + k + 64 * g + 16 * u);
        acc[j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fb[buf][u], x, acc[j], 0, 0, 0);
      }
    }
  }
  __device__ __forceinline__ void run() {
    const int n = rounds();
    for (int i = wave; i < n; i += 2 * W) {
      if (i + W < n) load(1, (i + W) * 64 * U);
      products(0, i * 64 * U);
      if (i + W < n) {
        if (i + 2 * W < n) load(0, (i + 2 * W) * 64 * U);
        products(1, (i + W) * 64 * U);
      }
    }
    if (wave == W - 1) {  // the rest of the sum, zeros past K on the weights' side
      for (int k = n * 64 * U; k < K; k += 64) {
        const int left = K - (k + 16 * g);
        i32x4 w = {0, 0, 0, 0}, y[R];
#pragma unroll
        for (int j = 0; j < R; ++j) y[j] = w;
        if (left > 0) {
          w = *reinterpret_cast<const i32x4*>(rb + k + 16 * g);
#pragma unroll
          for (int j = 0; j < R; ++j) y[j] = *reinterpret_cast<const i32x4*>(ra[j] + k + 16 * g);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int m = left - 4 * e;  // bytes of this word that belong to the sum
          if (m < 4) w[e] = m <= 0 ? 0 : w[e] & (int)((1u << (8 * m)) - 1u);
        }
#pragma unroll
        for (int j = 0; j < R; ++j) acc[j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w, y[j], acc[j], 0, 0, 0);
      }
    }
  }
  // the wavefronts' sums together and the results out, group j by wavefront j; sa: the scale of an activation row
  template <typename TO, typename SA>
  __device__ __forceinline__ void finish(const LinearArgs& a, int64_t n0, i32x4 (*part)[R][64], const SA& sa) {
#pragma unroll
    for (int j = 0; j < R; ++j) part[wave][j][lane] = acc[j];
    __syncthreads();
    const int64_t m = 16 * wave + (lane & 15), n = n0 + 4 * g;
    if (wave >= R || m >= a.M) return;
    i32x4 sum = part[0][wave][lane];
#pragma unroll
    for (int w = 1; w < W; ++w) sum += part[w][wave][lane];
    const float s = sa(m);
    float y[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int64_t nn = n + e < a.N ? n + e : a.N - 1;
      y[e] = scaled(sum[e], s, a.b_scale[nn], a.bias ? a.bias[nn] : 0.0f);
    }
    TO* o = static_cast<TO*>(a.out) + m * a.ldo;
    store4(o, y, n, a.N, ((reinterpret_cast<uintptr_t>(a.out) | (uintptr_t)(a.ldo * sizeof(TO))) & (4 * sizeof(TO) - 1)) == 0);
  }
};

// On activation codes in memory.  Weights in the last cache: 13 x 2560 x 2048 3.2 us, 13 x 2048 x 11008 7.7
// (128 workgroups: half of the CUs at 23 GB/s of weights each, 2.9 TB/s in all); from memory the latter takes 10.2.
template <int W, int R, typename TO>
__global__ __launch_bounds__(64 * W) void k_matmul_i8_rows(LinearArgs a) {
  __shared__ i32x4 part[W][R][64];
  const int64_t n0 = (int64_t)blockIdx.x * 16;
  RowSums<W, R, true> sums(a, n0, threadIdx.x & 63, threadIdx.x >> 6, a.A, a.lda);
  sums.begin();
  sums.run();
  sums.template finish<TO>(a, n0, part, [&](int64_t m) { return a.a_scale[m]; });
}

// On activations: every workgroup quantizes the few rows itself (into LDS, as
// quant_i8.hip does), while its first weights are on their way, which saves a
// launch and its wait.  Each row's values are read twice, the second time from
// the nearest cache.  Bound by latency: 1 x 2560 x 2048 4.5 us, 5.0 with weights from memory, of which the 5 MB take 0.8.
template <int W, typename T, typename TO>
__global__ __launch_bounds__(64 * W) void k_linear_i8_rows(LinearArgs a, const T* X, int64_t ldx, int pitch, bool wide) {
  __shared__ i32x4 part[W][1][64];
  __shared__ float peak[W];
  __shared__ float scales[16];
  extern __shared__ __attribute__((aligned(16))) int8_t codes[];  // [M][pitch]
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t n0 = (int64_t)blockIdx.x * 16;
  RowSums<W, 1, false> sums(a, n0, lane, wave, codes, pitch);
  sums.begin();
  const int M = (int)a.M, K = (int)a.K;
  // G wavefronts a row, W / G rows at once
  const int G = M <= 1 ? W : M <= 2 ? W / 2 : M <= 4 ? W / 4 : 1;
  const int sub = wave & (G - 1), t = sub * 64 + lane;
  for (int base = 0; base < M; base += W / G) {
    const int m = base + wave / G;
    const bool live = m < M;
    const T* x = X + (live ? m : 0) * ldx;
    float top = 0.0f;
    if (live)
#pragma unroll 4
      for (int at = t * 8; at < K; at += G * 512) {
        float v[8];
        load8(x + at, K - at, wide, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) top = amax_keep(top, v[e]);
      }
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) top = amax_keep(top, __shfl_xor(top, off, 64));
    if (G > 1) {
      if (lane == 0) peak[wave] = top;
      __syncthreads();
      for (int w = 0; w < G; ++w) top = amax_keep(top, peak[(wave & ~(G - 1)) + w]);
      __syncthreads();
    }
    const float s = scale_of_amax(top);
    const float inv = inverse_scale(s);
    if (live) {
#pragma unroll 4
      for (int at = t * 8; at < pitch; at += G * 512) {
        float v[8];
        load8(x + at, K - at, wide, v);
        *reinterpret_cast<uint2*>(codes + m * pitch + at) = codes8(v, inv, s == s);
      }
      if (t == 0) scales[m] = s;
    }
  }
  __syncthreads();
  sums.run();
  sums.template finish<TO>(a, n0, part, [&](int64_t m) { return scales[m]; });
}

// Tiles through LDS, for products with enough rows to fill the matrix cores.
//
// A workgroup makes BM rows (m) times BN columns (n) of the result, a
// wavefront WM x WN of them as 32 x 32 tiles of v_mfma_i32_32x32x32_i8.  The sum
// advances 128 bytes at a time through two to four LDS stages filled by direct
// global-to-LDS loads, which leave the registers to the sums.  A stage's rows
// of 128 bytes are 8 pieces of 16; piece p of row r lies at place p ^ key(r).  LDS
// serves 16 lanes a cycle (64 banks), two rows side by side: over the 16 rows
// that a fragment read takes together, (row % 2, key) takes 16 values.  (Keys of
// 8 rows, row % 8, took twice the cycles.)  The fills of the next steps and the
// fragment reads of the next 32 bytes are issued before the products of the
// current ones.  Eight wavefronts of 128 x 64 make a 256 x 256 tile (four of
// 128 x 128 wait at every barrier together: 1.20 against 1.11 ms at 8192 x 27648
// x 5120; 1.06 with results that leave in whole lines, 2.19 POPS, where a library's
// product of the same matrices into int32 takes 1.11).  Bound by the matrix cores
// there, by the weights' bytes with few rows (64 x 27648 x 5120: 29.7 us, 4.9 TB/s),
// and by LDS and barriers a step where the tiles do not fill the machine.
//
// Rows and pieces past the operands' ends come from beyond the buffer resource
// and arrive as zeros.  Where K is no multiple of 16 the bytes past it are
// cleared in LDS, on A's side alone (0 times whatever B holds).
//
// Weight row 8 b + 4 h + i of a 32-row tile carries column 16 h + 4 b + i, so
// that a lane (half h) ends with 16 consecutive columns of one result row.
constexpr int kStep = 128;

__device__ __forceinline__ int key_a(int row) { return (row >> 1) & 7; }
__device__ __forceinline__ int key_b(int row) { return ((row >> 1) & 3) | ((row >> 2) & 4); }

// A barrier for LDS contents alone: __syncthreads() would also wait for every
// fill that is still to come.
__device__ __forceinline__ void sync_lds() {
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

template <int BM, int BN, int WM, int WN>
struct TileShape {
  static constexpr int kWaves = (BM / WM) * (BN / WN);
  static constexpr int kThreads = 64 * kWaves;
  static constexpr int kStage = (BM + BN) * kStep;
};

template <int BM, int BN, int WM, int WN, int OCC, int NS, bool ONCE, typename TO>
__global__ __launch_bounds__((TileShape<BM, BN, WM, WN>::kThreads), OCC) void k_matmul_i8_tile(LinearArgs a, int tiles_m,
                                                                                               int tiles_n,
                                                                                               int split_steps,
                                                                                               int32_t* parts) {
  using S = TileShape<BM, BN, WM, WN>;
  constexpr int TM = WM / 32, TN = WN / 32;
  constexpr int NA = BM * 8 / S::kThreads, NB = BN * 8 / S::kThreads;  // 16-byte pieces per thread and step
  constexpr int kRows = S::kThreads / 8;                              // rows that one round of fills covers
  static_assert(kRows == 16 || kRows % 32 == 0, "keys of a round of fills");
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
  const uint32_t oa = (uint32_t)frow * (uint32_t)a.lda + pa, ob = (uint32_t)frow * (uint32_t)a.ldb;
  const uint32_t sa = kRows * (uint32_t)a.lda, sb = kRows * (uint32_t)a.ldb;
  typedef __attribute__((address_space(3))) void* lds_ptr;
  const int first = (int)blockIdx.y * split_steps;  // this workgroup's steps of the sum
  const int all = (K + kStep - 1) / kStep;
  const int steps = all - first < split_steps ? all - first : split_steps;
  auto fill = [&](int stage, int t) {
    const int k = t < steps ? (first + t) * kStep : K;
    char* base = lds + stage * S::kStage + wave * 1024;
    const bool ina = k + pa < K;
#pragma unroll
    for (int i = 0; i < NA; ++i)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(ra, (lds_ptr)(base + i * kRows * kStep), 16,
                                               ina ? (int)(oa + i * sa + k) : (int)0x80000000, 0, 0, 0);
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      // rows 16 on have bit 2 of the key flipped
      const int p = kRows == 16 && (i & 1) ? pb ^ 64 : pb;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rb, (lds_ptr)(base + (BM + i * kRows) * kStep), 16,
                                               k + p < K ? (int)(ob + i * sb + p + k) : (int)0x80000000, 0, 0, ONCE ? 2 : 0);
    }
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

  // waits until step t's fills are in, this wavefront's and then everyone's (LATER fills follow them); clears what lies
  // past K in A's rows of the last step
  auto arrived = [&](auto later, int stage, int t) {
    constexpr int n = decltype(later)::value * (NA + NB);
    static_assert(n < 64, "vmcnt");
    __builtin_amdgcn_s_waitcnt(0x0F70 | (n & 15) | (n >> 4) << 14);  // vmcnt(n)
    sync_lds();                                                    // (every fragment of the stage that is refilled next is read)
    if (first + t == all - 1 && K != K16) {
      const int k = K - (K16 - 16), p = (K16 - 16 - (first + t) * kStep) >> 4;
      for (int row = tid; row < BM; row += S::kThreads) {
        char* c = lds + stage * S::kStage + row * kStep + (p ^ key_a(row)) * 16;
        for (int e = k; e < 16; ++e) c[e] = 0;
      }
      sync_lds();
    }
  };

  // fills past the last step come from beyond the resources: they keep the counts and read nothing
#pragma unroll
  for (int t = 0; t < NS; ++t) fill(t, t);
  arrived(std::integral_constant<int, NS - 1>{}, 0, 0);
  int st = 0;
  if constexpr (TM * TN == 1) {
    // One product for two fragments: a whole step's are read during the products of the step before (read 32 bytes
    // ahead, as below, each product waits for LDS: 100 x 5120 x 5120 15.4 us, 13.9; tiles of more products gain nothing).
    i32x4 fa[2][4][TM], fb[2][4][TN];
    const auto read = [&](int stage, int b) {
#pragma unroll
      for (int ks = 0; ks < 4; ++ks) frags(stage, ks, fa[b][ks], fb[b][ks]);
    };
    read(0, 0);
    for (int t0 = 0; t0 < steps; t0 += 2) {
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const int t = t0 + b;
        if (t >= steps) break;
        const int next = st + 1 == NS ? 0 : st + 1;
        arrived(std::integral_constant<int, NS - 2>{}, next, t + 1);
        fill(st, t + NS);
        read(next, b ^ 1);
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) products(fa[b][ks], fb[b][ks]);
        st = next;
      }
    }
  } else {
    i32x4 fa[2][TM], fb[2][TN];
    frags(0, 0, fa[0], fb[0]);
    // the order of a phase: the fragment reads, and in the last phase the fills after them, between the products that
    // hide them (left alone the compiler waits for reads right after it issues them)
    const auto order = [&](auto fills) {
      constexpr bool kFills = decltype(fills)::value;
      constexpr int n_mfma = TM * TN, n_read = TM + TN, n_fill = kFills ? NA + NB : 0;
      constexpr int per = kFills || n_mfma < 2 * n_read ? 1 : n_mfma / n_read;
#pragma unroll
      for (int i = 0; i < n_read; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, per, 0);  // MFMA
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);    // LDS read
      }
      if constexpr (kFills) {
        constexpr int left = n_mfma - n_read > 0 ? n_mfma - n_read : 1;
#pragma unroll
        for (int i = 0; i < left; ++i) {
          __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
          __builtin_amdgcn_sched_group_barrier(0x020, (n_fill + left - 1) / left, 0);  // memory read
        }
      }
    };
    for (int t = 0; t < steps; ++t) {
#pragma unroll
      for (int ks = 0; ks < 3; ++ks) {
        frags(st, ks + 1, fa[(ks + 1) & 1], fb[(ks + 1) & 1]);
        products(fa[ks & 1], fb[ks & 1]);
        order(std::false_type{});
      }
      const int next = st + 1 == NS ? 0 : st + 1;
      arrived(std::integral_constant<int, NS - 2>{}, next, t + 1);
      fill(st, t + NS);
      frags(next, 0, fa[0], fb[0]);
      products(fa[1], fb[1]);
      order(std::true_type{});
      st = next;
    }
  }
  __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0): no fill outlives the workgroup

  // results: lane -> row wm + 32 j + r, columns wn + 32 i + 16 half + e
  if (parts) {  // a part of the sum, for k_matmul_i8_join
    int32_t* o = parts + (int64_t)blockIdx.y * a.M * a.N;
#pragma unroll
    for (int i = 0; i < TN; ++i)
#pragma unroll
      for (int j = 0; j < TM; ++j) {
        const int64_t m = m0 + wm + 32 * j + r, n = n0 + wn + 32 * i + 16 * half;
        if (m >= a.M) continue;
        if (n + 16 <= a.N && (a.N & 3) == 0) {
#pragma unroll
          for (int e = 0; e < 16; e += 4)
            *reinterpret_cast<i32x4*>(o + m * a.N + n + e) =
                i32x4{acc[i][j][e], acc[i][j][e + 1], acc[i][j][e + 2], acc[i][j][e + 3]};
        } else {
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (n + e < a.N) o[m * a.N + n + e] = acc[i][j][e];
        }
      }
    return;
  }
  const bool wide = ((reinterpret_cast<uintptr_t>(a.out) | (uintptr_t)(a.ldo * sizeof(TO))) & 15) == 0;
  float sav[TM];
#pragma unroll
  for (int j = 0; j < TM; ++j) {
    const int64_t m = m0 + wm + 32 * j + r;
    sav[j] = a.a_scale[m < a.M ? m : a.M - 1];
  }
  // Results go out by groups of 64 or 128 bytes of a row: through the wavefront's own part of LDS (the stages are done
  // with), so that a store covers whole lines instead of a piece of each of 64 (5971 x 7503 x 4953 into fp32 rows that
  // do not lie on 16 bytes: 417 us with plain stores of single values, 288).
  constexpr int GT = WN * sizeof(TO) >= 128 && sizeof(TO) == 2 ? 2 : 1;  // 32-column tiles of a group
  constexpr int V = 16 / sizeof(TO), kPieces = 32 * GT / V;              // values of a piece, pieces of a group's row
  static_assert(WM * kPieces * 16 * S::kWaves <= NS * S::kStage, "LDS of the results");
  typedef TO Piece __attribute__((ext_vector_type(16 / sizeof(TO))));
  char* mine = lds + wave * (WM * kPieces * 16);
  __syncthreads();
#pragma unroll
  for (int i0 = 0; i0 < TN; i0 += GT) {
#pragma unroll
    for (int i = i0; i < i0 + GT; ++i) {
      const int64_t n = n0 + wn + 32 * i + 16 * half;
      float sbv[16], bias[16];
      if (n0 + wn + 32 * (i + 1) <= a.N && (reinterpret_cast<uintptr_t>(a.b_scale) & 15) == 0 &&
          (reinterpret_cast<uintptr_t>(a.bias) & 15) == 0) {
#pragma unroll
        for (int e = 0; e < 16; e += 4) {
          const fl4 x = *reinterpret_cast<const fl4*>(a.b_scale + n + e);
          const fl4 y = a.bias ? *reinterpret_cast<const fl4*>(a.bias + n + e) : fl4{0, 0, 0, 0};
#pragma unroll
          for (int f = 0; f < 4; ++f) {
            sbv[e + f] = x[f];
            bias[e + f] = y[f];
          }
        }
      } else {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int64_t nn = n + e < a.N ? n + e : a.N - 1;
          sbv[e] = a.b_scale[nn];
          bias[e] = a.bias ? a.bias[nn] : 0.0f;
        }
      }
#pragma unroll
      for (int j = 0; j < TM; ++j) {
        const int row = 32 * j + r;
#pragma unroll
        for (int p = 0; p < 16 / V; ++p) {
          Piece w;
#pragma unroll
          for (int e = 0; e < V; ++e) w[e] = (TO)scaled(acc[i][j][p * V + e], sav[j], sbv[p * V + e], bias[p * V + e]);
          const int at = (32 * (i - i0) + 16 * half) / V + p;
          *reinterpret_cast<Piece*>(mine + (row * kPieces + (at ^ (row & (kPieces - 1)))) * 16) = w;
        }
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    TO* o = static_cast<TO*>(a.out) + (m0 + wm) * a.ldo + n0 + wn + 32 * i0;
    if (wide && n0 + wn + 32 * (i0 + GT) <= a.N) {
#pragma unroll
      for (int p = 0; p < WM * kPieces / 64; ++p) {
        const int x = p * 64 + lane, row = x / kPieces, at = x % kPieces;
        const Piece w = *reinterpret_cast<const Piece*>(mine + (row * kPieces + (at ^ (row & (kPieces - 1)))) * 16);
        if (m0 + wm + row < a.M) *reinterpret_cast<Piece*>(o + row * a.ldo + at * V) = w;
      }
    } else {  // rows that do not lie on 16 bytes, or the last columns
      const int64_t left = a.N - (n0 + wn + 32 * i0);
#pragma unroll 4
      for (int p = 0; p < WM * GT / 2; ++p) {
        const int x = p * 64 + lane, row = x / (32 * GT), col = x % (32 * GT);
        const char* w = mine + (row * kPieces + ((col / V) ^ (row & (kPieces - 1)))) * 16 + col % V * sizeof(TO);
        if (m0 + wm + row < a.M && col < left) o[row * a.ldo + col] = *reinterpret_cast<const TO*>(w);
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  }
}

// The parts of split sums together, with the epilogue; four columns a thread.  A few us of latency: 64 x 2048 in 5 parts, 2.6 MB.
template <typename TO>
__global__ __launch_bounds__(256) void k_matmul_i8_join(LinearArgs a, const int32_t* __restrict__ parts, int n_parts) {
  const int64_t quads = (a.N + 3) / 4;
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= quads * a.M) return;
  const int64_t m = i / quads, n = (i - m * quads) * 4;
  int sum[4] = {0, 0, 0, 0};
  for (int p = 0; p < n_parts; ++p) {
    const int32_t* s = parts + ((int64_t)p * a.M + m) * a.N + n;
    if ((a.N & 3) == 0) {
      const i32x4 v = *reinterpret_cast<const i32x4*>(s);
#pragma unroll
      for (int e = 0; e < 4; ++e) sum[e] += v[e];
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) sum[e] += n + e < a.N ? s[e] : 0;
    }
  }
  const float sa = a.a_scale[m];
  float y[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int64_t nn = n + e < a.N ? n + e : a.N - 1;
    y[e] = scaled(sum[e], sa, a.b_scale[nn], a.bias ? a.bias[nn] : 0.0f);
  }
  TO* o = static_cast<TO*>(a.out) + m * a.ldo;
  store4(o, y, n, a.N, ((reinterpret_cast<uintptr_t>(a.out) | (uintptr_t)(a.ldo * sizeof(TO))) & (4 * sizeof(TO) - 1)) == 0);
}

template <int BM, int BN, int WM, int WN, int OCC, int NS, bool ONCE, typename TO>
hipError_t launch_tile(const LinearArgs& a, int split, void* ws, hipStream_t st) {
  using S = TileShape<BM, BN, WM, WN>;
  const auto k = k_matmul_i8_tile<BM, BN, WM, WN, OCC, NS, ONCE, TO>;
  const size_t lds = NS * S::kStage;
  if (lds > 65536) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(k), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return e;
  }
  const int64_t tm = (a.M + BM - 1) / BM, tn = (a.N + BN - 1) / BN;
  if (tm * tn > 0x7FFFFFFF / S::kThreads) return hipErrorInvalidValue;  // (threads of a launch: more than memory holds results for)
  const int all = (int)((a.K + kStep - 1) / kStep), per = (all + split - 1) / split;
  split = (all + per - 1) / per;
  int32_t* parts = split > 1 ? static_cast<int32_t*>(ws) : nullptr;
  hipLaunchKernelGGL(k, dim3((unsigned)(tm * tn), (unsigned)split), dim3(S::kThreads), lds, st, a, (int)tm, (int)tn, per, parts);
  if (parts) {
    const int64_t quads = a.M * ((a.N + 3) / 4);
    hipLaunchKernelGGL((k_matmul_i8_join<TO>), dim3((unsigned)((quads + 255) / 256)), dim3(256), 0, st, a, parts, split);
  }
  return hipGetLastError();
}

// Bytes between rows of codes in LDS: whole steps, and 16 more so that rows start in different banks.
int linear_rows_pitch(int64_t K) { return (int)((K + 63) / 64 * 64 + 16); }

template <int W, int R, typename TO>
hipError_t launch_rows(const LinearArgs& a, hipStream_t st) {
  hipLaunchKernelGGL((k_matmul_i8_rows<W, R, TO>), dim3((unsigned)((a.N + 15) / 16)), dim3(64 * W), 0, st, a);
  return hipGetLastError();
}

template <int W, typename T, typename TO>
hipError_t launch_linear_rows(const LinearArgs& a, const void* X, int64_t ldx, hipStream_t st) {
  const bool wide = ((reinterpret_cast<uintptr_t>(X) | (uintptr_t)(ldx * sizeof(T))) & 15) == 0;
  const int pitch = linear_rows_pitch(a.K);
  hipLaunchKernelGGL((k_linear_i8_rows<W, T, TO>), dim3((unsigned)((a.N + 15) / 16)), dim3(64 * W), (size_t)a.M * pitch, st, a,
                     static_cast<const T*>(X), ldx, pitch, wide);
  return hipGetLastError();
}
template <int W, typename T>
hipError_t launch_linear_rows_w(const LinearArgs& a, const void* X, int64_t ldx, hipStream_t st) {
  if (a.out_dtype == AWSRC_DTYPE_F32) return launch_linear_rows<W, T, float>(a, X, ldx, st);
  if (a.out_dtype == AWSRC_DTYPE_BF16) return launch_linear_rows<W, T, __bf16>(a, X, ldx, st);
  return launch_linear_rows<W, T, _Float16>(a, X, ldx, st);
}
template <typename T>
hipError_t launch_linear_rows_t(const LinearArgs& a, const void* X, int64_t ldx, hipStream_t st) {
  // more than 8 rows: as many wavefronts, each quantizing one (16 x 2048 x 2048: 7.7 us, 9.8 with 8)
  return a.M <= 8 ? launch_linear_rows_w<8, T>(a, X, ldx, st) : launch_linear_rows_w<16, T>(a, X, ldx, st);
}

// Which kernel takes a product, and over how many parts of the sum.  Times below
// are in us, of calls on weights that are not in the caches.
enum Path { kRows, kTile32, kTile64, kTile64Wide, kTile128, kTile256 };
struct Choice {
  Path path;
  int split;
};
Choice choose(int64_t M, int64_t N, int64_t K) {
  const auto tiles = [&](int64_t bm, int64_t bn) { return ((M + bm - 1) / bm) * ((N + bn - 1) / bn); };
  // Up to 16 rows: 16 columns a workgroup, up to about three of them a CU (16 x 11008 x
  // 2048: 6.9, through LDS tiles 8.1); with more the activations' reads, as many bytes as
  // the weights', cost more than tiles do (16 x 13824 x 5120: 18.3 and 17.2; 16 x 27648 x
  // 5120: 32.4 and 28.1).  Loads past the last cache do not pay here (16 x 8192 x 8192: 15.2, 13.0 without).
  if (M <= 16 && N < 12288) return {kRows, 1};
  // Up to 32 rows of them while the sum is not so long that its parts pay (30 x 2560 x 2048: 3.9, tiles 6.6; 32 x 4096 x
  // 4096: 6.6 and 10.0; 24 x 5120 x 5120: 11.3 and 11.1; 32 x 8192 x 8192: 17.1 and 23.4; 32 x 11008 x 2048: 9.4 and 7.5;
  // 32 x 4096 x 27648: 33.8 and 26.0).
  if (M > 16 && M <= 32 && N <= 8192 && K <= 16384) return {kRows, 1};
  // 256 tiles of 128 cost 24 us at K = 5120, a round of 256 tiles of 256, one per CU, 62
  // to 80 (512 x 27648 x 5120: 117 and 93; 4096 x 5120 x 5120, two rounds, 117 and 123;
  // 1024 x 5120 x 5120: 40 and 54; 8192 x 27648 x 5120: 1249 and 1105).
  const int64_t t128 = tiles(128, 128), t256 = tiles(256, 256);
  if (M > 64 && t128 >= 256) return {2.9 * ((t256 + 255) / 256) < t128 / 256.0 + 0.5 ? kTile256 : kTile128, 1};
  // 64 x 27648 x 5120: 64 x 64 tiles 37.7, 64 x 128 tiles 29.7 (64 x 11008 x 2048: 7.8 and 10.5)
  if (M > 32 && tiles(64, 128) >= 192) return {kTile64Wide, 1};
  const Path path = M > 32 ? kTile64 : kTile32;
  // Few tiles under a long sum: parts of at least 16 steps, joined by a second
  // launch (64 x 2048 x 11008: 28 whole, 13.4 in 5 parts; 64 x 2560 x 2048: 6.7 whole, 8.9 in 4)
  const int64_t t = path == kTile64 ? tiles(64, 64) : tiles(32, 64);
  const int64_t want = (256 + t - 1) / t, most = (K + kStep - 1) / kStep / 16;
  const int64_t split = want < most ? want : most;
  return {path, t < 128 && split > 1 ? (int)split : 1};
}

template <typename TO>
hipError_t launch(const LinearArgs& a, void* ws, hipStream_t st) {
  const Choice c = choose(a.M, a.N, a.K);
  // Weights read once that fill a good part of the last cache go past it (64 x 27648 x 5120: 33.0 us, 29.7 past
  // it; 16 x 27648 x 5120 30.3 and 26.6; 64 x 11008 x 2048, whose 23 MB stay there from call to call: 8.8, 10.1 past
  // it).  64 x 64 tiles, of fewer columns, keep theirs: not tried there.
  const bool once = a.M <= 64 && a.N * a.K >= (int64_t)1 << 26;
  switch (c.path) {
    case kRows: return a.M <= 16 ? launch_rows<8, 1, TO>(a, st) : launch_rows<8, 2, TO>(a, st);
    case kTile32:
      return once ? launch_tile<32, 64, 32, 32, 2, 4, true, TO>(a, c.split, ws, st)
                  : launch_tile<32, 64, 32, 32, 2, 4, false, TO>(a, c.split, ws, st);
    case kTile64: return launch_tile<64, 64, 32, 32, 2, 4, false, TO>(a, c.split, ws, st);
    case kTile64Wide:
      return once ? launch_tile<64, 128, 32, 64, 2, 3, true, TO>(a, 1, ws, st)
                  : launch_tile<64, 128, 32, 64, 2, 3, false, TO>(a, 1, ws, st);
    case kTile128: return launch_tile<128, 128, 64, 64, 2, 2, false, TO>(a, 1, ws, st);
    default: return launch_tile<256, 256, 128, 64, 2, 2, false, TO>(a, 1, ws, st);
  }
}

}  // namespace

size_t matmul_i8_ws_bytes(int64_t M, int64_t N, int64_t K) {
  const int split = choose(M, N, K).split;
  return split > 1 ? (size_t)split * (size_t)M * (size_t)N * 4 : 0;
}

hipError_t launch_matmul_i8(const LinearArgs& a, void* ws, hipStream_t st) {
  if (a.out_dtype == AWSRC_DTYPE_F32) return launch<float>(a, ws, st);
  if (a.out_dtype == AWSRC_DTYPE_BF16) return launch<__bf16>(a, ws, st);
  return launch<_Float16>(a, ws, st);
}

bool linear_i8_fused(int64_t M, int64_t N, int64_t K) {
  // Where a workgroup's wavefronts read the rows in few pieces a lane, and where there are not so many
  // workgroups that quantizing over and over costs more than a launch.  On the GPU alone, in us (fused and in two
  // launches): 1 x 2560 x 2048 4.5 and 5.7; 1 x 5120 x 5120 8.9 and 10.9; 4 x 5120 x 4096 11.8 and 10.4;
  // 16 x 2048 x 2048 7.7 and 6.0; 1 x 27648 x 5120 31.6 and 28.9.  A launch that is not
  // replayed from a graph costs the host 3 more, which is why the middle ones are fused.  From 8192 columns a call has
  // a workspace to give and takes two launches, also where fusing up to 12288 would gain on the GPU (1 x 11008 x 2048:
  // 8.7 and 10.7; 4 x 11008 x 2048 10.4 and 10.9).
  const int64_t share = M <= 1 ? 1 : M <= 2 ? 2 : M <= 4 ? 4 : 8;
  return M <= 16 && K * share <= 16384 && N < 8192;
}

hipError_t launch_linear_i8_fused(const LinearArgs& a, const void* X, int x_dtype, int64_t ldx, hipStream_t st) {
  if (x_dtype == AWSRC_DTYPE_F32) return launch_linear_rows_t<float>(a, X, ldx, st);
  if (x_dtype == AWSRC_DTYPE_BF16) return launch_linear_rows_t<__bf16>(a, X, ldx, st);
  return launch_linear_rows_t<_Float16>(a, X, ldx, st);
}

}  // namespace awsrc
