// Products of e4m3 matrices with a scale for each block of 128:
//   out[m][n] = sum_b a_scale[b][m] b_scale[n / 128][b] sum_{k in b} A[m][k] B[n][k] + bias[n].
// Four v_mfma_f32_16x16x32_f16 from a zero accumulator are a block's sums of
// a 16 x 16 tile; one fma a value then adds them with their scale.  The codes go as
// fp16, which holds them exactly.
//
// The matrix cores take e4m3 as well, at twice the rate, but then they add eight adjacent products
// at the exponent of the largest and cut off what lies 2^13 below it (measured, of
// v_mfma_f32_16x16x128_f8f6f4 and v_mfma_f32_16x16x32_fp8_fp8 alike): random codes come out 1.5e-5 to 5e-5
// rms off, and products that a louder neighbour hides are lost where the loud ones cancel.  In fp16
// they add in fp32: whole numbers below 2^24 exactly, random codes within 8e-8 rms.
//
// Matrix-core layout: an operand lane l holds row l % 16 and 32 bytes of a block
// of 128, the same ones in both operands; the result
// lane holds column l % 16 and rows 4 (l / 16) + i.  B (the weights) takes the rows'
// place and A the columns', so that a lane ends with four consecutive n of one m,
// and with one scale of A.
#include <type_traits>
#include "serve_internal.h"

namespace awsrc {

namespace {

// Eight codes as fp16.
__device__ __forceinline__ h8 halves(int lo, int hi) {
  const auto a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((uint32_t)lo, 1.0f, false);
  const auto b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((uint32_t)lo, 1.0f, true);
  const auto c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((uint32_t)hi, 1.0f, false);
  const auto d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((uint32_t)hi, 1.0f, true);
  return h8{(_Float16)a[0], (_Float16)a[1], (_Float16)b[0], (_Float16)b[1],
            (_Float16)c[0], (_Float16)c[1], (_Float16)d[0], (_Float16)d[1]};
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

// An operand's 32 bytes as the products take them.
struct Operand {
  h8 v[4];
  __device__ __forceinline__ void set(i32x4 lo, i32x4 hi) {
    v[0] = halves(lo[0], lo[1]);
    v[1] = halves(lo[2], lo[3]);
    v[2] = halves(hi[0], hi[1]);
    v[3] = halves(hi[2], hi[3]);
  }
};
__device__ __forceinline__ fl4 sums_of(const Operand& w, const Operand& x) {
  fl4 p = {0, 0, 0, 0};
#pragma unroll
  for (int i = 0; i < 4; ++i) p = __builtin_amdgcn_mfma_f32_16x16x32_f16(w.v[i], x.v[i], p, 0, 0, 0);
  return p;
}

// Up to 16 rows (or 32: R groups of 16): the weights' bytes are all that counts.  A workgroup takes 16
// weight rows (columns of the result) against all activation rows, its W
// wavefronts sharing the sum; the weights come straight from memory, two blocks
// ahead of the products, and the wavefronts' sums meet in LDS.
//
// The matrix cores want a lane to hold 32 bytes of its own row, but a CU's cache
// takes in a quad of lanes a cycle only where they read 64 bytes side by side.  So
// lane j of a quad loads piece j of its quad's four rows, and the quad trades them:
// a lane of group g = lane / 16 ends with 64 bytes of its row, the first half of block 0,
// of block 1, the second half of block 0 and of block 1 for g = 0 to 3.  Groups 0 and 1, 2 and 3
// trade halves of those with one instruction a register: 32 bytes of each block.
//
// 13 x 2048 x 11008 (23 MB): 8.3 us with the weights in the caches, 11.7 from memory, of which 3.7 are their
// bytes: 128 workgroups do not keep enough on its way for more.
struct Quads {
  static constexpr int kRound = 2 * kBlockF8;  // bytes of a row that a wavefront takes at a time
  i32x4 v[4];
  // `row` gives a row's address; the lane loads piece lane % 4 of rows 4 (lane % 16 / 4) + u
  template <typename F>
  static __device__ __forceinline__ void pointers(const uint8_t* (&p)[4], int lane, const F& row) {
    const int g = lane >> 4;
#pragma unroll
    for (int u = 0; u < 4; ++u) p[u] = row((lane & 12) + u) + ((g & 1) * kBlockF8 + (g >> 1) * 64) + 16 * (lane & 3);
  }
  template <bool ONCE>  // past the caches
  __device__ __forceinline__ void load(const uint8_t* const (&p)[4], int k) {
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const i32x4* w = reinterpret_cast<const i32x4*>(p[u] + k);
      v[u] = ONCE ? __builtin_nontemporal_load(w) : *w;
    }
  }
  // the quads trade, then the groups
  __device__ __forceinline__ void turn(int lane, Operand& block0, Operand& block1) {
    turn_quads(v, lane);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {  // odd groups' first half against even groups' second half
        const auto t = __builtin_amdgcn_permlane16_swap((uint32_t)v[i][e], (uint32_t)v[i + 2][e], false, false);
        v[i][e] = (int)t[0];
        v[i + 2][e] = (int)t[1];
      }
    }
    block0.set(v[0], v[1]);
    block1.set(v[2], v[3]);
  }
};

template <int W, int R, bool AHEAD, bool ONCE, typename TO>
struct RowSums {
  const uint8_t* pb[4];      // this lane's pieces of the weights
  const uint8_t* pa[R][4];   // the same of R groups of 16 rows of activation codes (AHEAD: in memory, fetched with the weights)
  const uint8_t *rb, *ra[R]; // this lane's own rows
  const float* sb;           // the weights' scales of this workgroup's columns
  int K, wave, lane, g;
  fl4 acc[R];
  Quads fb[2], fa[2][R];

  // rows that do not exist read the last one: their sums are not stored
  __device__ __forceinline__ RowSums(const LinearF8Args& a, int64_t n0, int ln, int wv, const uint8_t* A, int64_t lda)
      : K((int)a.K), wave(wv), lane(ln), g(ln >> 4) {
    const auto weights = [&](int r) { return a.B + (n0 + r < a.N ? n0 + r : a.N - 1) * a.ldb; };
    Quads::pointers(pb, ln, weights);
    rb = weights(ln & 15);
    sb = a.b_scale + n0 / kBlockF8 * ((a.K + kBlockF8 - 1) / kBlockF8);
#pragma unroll
    for (int j = 0; j < R; ++j) {
      const auto codes = [&](int r) { return A + (16 * j + r < a.M ? 16 * j + r : a.M - 1) * lda; };
      Quads::pointers(pa[j], ln, codes);
      ra[j] = codes(ln & 15);
      acc[j] = fl4{0, 0, 0, 0};
    }
  }
  __device__ __forceinline__ void load(int buf, int k) {
    fb[buf].template load<ONCE>(pb, k);
    if constexpr (AHEAD)
#pragma unroll
      for (int j = 0; j < R; ++j) fa[buf][j].template load<false>(pa[j], k);
  }
  __device__ __forceinline__ int rounds() const { return K / Quads::kRound; }
  __device__ __forceinline__ void begin() {
    if (wave < rounds()) load(0, wave * Quads::kRound);
  }
  __device__ __forceinline__ void add(int j, const Operand& w, const Operand& x, float s) {
    const fl4 p = sums_of(w, x);
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[j][e] = __builtin_fmaf(p[e], s, acc[j][e]);
  }
  template <typename SA>
  __device__ __forceinline__ void products(int buf, int k, const SA& sa) {
    const int b = k / kBlockF8;
    Operand w[2];
    fb[buf].turn(lane, w[0], w[1]);
#pragma unroll
    for (int j = 0; j < R; ++j) {
      Operand x[2];
      if constexpr (AHEAD) {
        fa[buf][j].turn(lane, x[0], x[1]);
      } else {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const uint8_t* c = ra[j] + k + h * kBlockF8 + 32 * g;
          x[h].set(*reinterpret_cast<const i32x4*>(c), *reinterpret_cast<const i32x4*>(c + 16));
        }
      }
#pragma unroll
      for (int h = 0; h < 2; ++h) add(j, w[h], x[h], sa(b + h, 16 * j + (lane & 15)) * sb[b + h]);
    }
  }
  // sa(b, m): the scale of block b of activation row m (of any row where m is none)
  template <typename SA>
  __device__ __forceinline__ void run(const SA& sa) {
    const int n = rounds();
    for (int i = wave; i < n; i += 2 * W) {
      if (i + W < n) load(1, (i + W) * Quads::kRound);
      products(0, i * Quads::kRound, sa);
      if (i + W < n) {
        if (i + 2 * W < n) load(0, (i + 2 * W) * Quads::kRound);
        products(1, (i + W) * Quads::kRound, sa);
      }
    }
    if (wave == W - 1) {  // the rest of the sum, zeros past K on both sides
      for (int k = n * Quads::kRound; k < K; k += kBlockF8) {
        const int at = k + 32 * g, left = K - at;
        Operand w;
        w.set(piece(rb + at, left), piece(rb + at + 16, left - 16));
#pragma unroll
        for (int j = 0; j < R; ++j) {
          Operand x;
          x.set(piece(ra[j] + at, left), piece(ra[j] + at + 16, left - 16));
          add(j, w, x, sa(k / kBlockF8, 16 * j + (lane & 15)) * sb[k / kBlockF8]);
        }
      }
    }
  }
  // the wavefronts' sums together and the results out, group j by wavefront j
  __device__ __forceinline__ void finish(const LinearF8Args& a, int64_t n0, fl4 (*part)[R][64]) {
#pragma unroll
    for (int j = 0; j < R; ++j) part[wave][j][lane] = acc[j];
    __syncthreads();
    const int64_t m = 16 * wave + (lane & 15), n = n0 + 4 * g;
    if (wave >= R || m >= a.M) return;
    fl4 sum = part[0][wave][lane];
#pragma unroll
    for (int w = 1; w < W; ++w) sum += part[w][wave][lane];
    float y[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int64_t nn = n + e < a.N ? n + e : a.N - 1;
      y[e] = rounded(sum[e] + (a.bias ? a.bias[nn] : 0.0f));
    }
    TO* o = static_cast<TO*>(a.out) + m * a.ldo;
    store4(o, y, n, a.N, ((reinterpret_cast<uintptr_t>(a.out) | (uintptr_t)(a.ldo * sizeof(TO))) & (4 * sizeof(TO) - 1)) == 0);
  }
};

// On activation codes in memory.
template <int W, int R, bool ONCE, typename TO>
__global__ __launch_bounds__(64 * W) void k_matmul_f8_rows(LinearF8Args a) {
  __shared__ fl4 part[W][R][64];
  const int64_t n0 = (int64_t)blockIdx.x * 16;
  RowSums<W, R, true, ONCE, TO> sums(a, n0, threadIdx.x & 63, __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), a.A, a.lda);
  sums.begin();
  sums.run([&](int b, int m) { return a.a_scale[(int64_t)b * a.M + (m < a.M ? m : a.M - 1)]; });
  sums.finish(a, n0, part);
}

// On activations: every workgroup quantizes the few rows itself (into LDS, as
// quant_f8.hip does, sixteen lanes a block), while its first weights are on their way, which saves a
// launch and its wait.  1 x 2560 x 2048 (5.3 MB) 4.3 us, 3.5 with the weights in the caches: one wait for X, one for the
// weights, and the wavefronts' meeting.
template <int W, bool ONCE, typename T, typename TO>
__global__ __launch_bounds__(64 * W) void k_linear_f8_rows(LinearF8Args a, const T* X, int64_t ldx, int pitch) {
  __shared__ fl4 part[W][1][64];
  extern __shared__ __attribute__((aligned(16))) uint8_t codes[];  // [M][pitch], then scales [blocks][16]
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t n0 = (int64_t)blockIdx.x * 16;
  RowSums<W, 1, false, ONCE, TO> sums(a, n0, lane, wave, codes, pitch);
  sums.begin();
  const int M = (int)a.M, K = (int)a.K, blocks = (K + kBlockF8 - 1) / kBlockF8;
  float* scales = reinterpret_cast<float*>(codes + M * pitch);
  const int at = (lane & 15) * 8;
  for (int i = threadIdx.x >> 4; i < M * blocks; i += 4 * W) {
    const int m = i / blocks, b = i - m * blocks, k = b * kBlockF8 + at;
    float v[8], top = 0.0f;
    load8_any(X + m * ldx + k, K - k, v);
#pragma unroll
    for (int e = 0; e < 8; ++e) top = amax_keep(top, v[e]);
    const float s = scale_of_amax_f8(amax_of_16(top));
    *reinterpret_cast<uint2*>(codes + m * pitch + k) = codes8_f8(v, inverse_scale(s), s > 0.0f);
    if (at == 0) scales[b * 16 + m] = s;
  }
  __syncthreads();
  sums.run([&](int b, int m) { return scales[b * 16 + (m < M ? m : M - 1)]; });
  sums.finish(a, n0, part);
}

// Tiles through LDS, for products with enough rows to fill the matrix cores.
//
// A workgroup makes BM rows (m) times BN columns (n) of the result, a
// wavefront WM x WN of them.  A step is a block of 128 of the sum: two or more LDS
// stages are filled by direct global-to-LDS loads, the codes and the block's scales of
// the tile's rows and columns.  A stage's rows of 128 bytes are 8 pieces of 16; piece p
// of row r lies at place p ^ key(r), and a lane takes pieces g and g + 4 of its row:
// over 16 lanes (row % 2, key) takes 16 values, which LDS serves without conflict.
//
// Rows past the operands' ends, and pieces that are not whole, come from beyond the buffer
// resource and arrive as zeros.  Where K is no multiple of 16 the rest of the sum, less than
// a piece, is added at the end straight from memory, zeros past K on both sides (a code
// there may be NaN).
//
// Weight row 4 TN q + 4 t + i of a wavefront's columns is row 4 q + i of its t-th
// operand, so that a lane ends with 4 TN consecutive columns of one result row.
//
// Bound by the matrix cores and by what stands beside them: the turn of codes into fp16 (sixteen
// instructions for an operand of a step) and an fma a value and block: matrix cores busy 57% of the time, vector units 68%.
// 8192 x 27648 x 5120 1.90 to 1.99 ms by machine, 1.2 PFLOP/s, as a library product of fp16 operands takes; 8192 x 8192 x 8192
// into fp32 0.91 ms, 1.21.  64 x 27648 x 5120 33.4 us (146 MB, 4.4 TB/s), 517 x 1003 x 1337 into
// fp32 11.2, of which the launch's latencies are most.
constexpr int kStep = kBlockF8;

__device__ __forceinline__ int key_a(int row) { return (row >> 1) & 7; }
template <int TN>
__device__ __forceinline__ int key_b(int row) { return ((row >> 1) & 1) | ((row / (4 * TN)) & 3) << 1; }

// An operand from a row on: the bytes up to its last readable one, as a buffer resource takes them; none past its rows.
struct Bytes {
  uint8_t* base;
  int size;
};
__device__ __forceinline__ Bytes bytes_from(const uint8_t* base, int64_t row, int64_t rows, int64_t ld, int cols) {
  const int64_t end = row < rows ? (rows - row - 1) * ld + cols : 0;
  return {const_cast<uint8_t*>(base + (row < rows ? row : 0) * ld), (int)(end < 0x7FFFFFFF ? end : 0x7FFFFFFF)};
}
// 16 bytes a lane from there to LDS, zeros past the end; ONCE: past the caches.
template <bool ONCE>
__device__ __forceinline__ void fill16(const Bytes& b, char* lds, int at) {
  const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(b.base, 0, b.size, 0x00020000);
  __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void*)lds, 16, at, 0, 0, ONCE ? 2 : 0);
}

template <int BM, int BN, int WM, int WN>
struct TileShape {
  static constexpr int kWaves = (BM / WM) * (BN / WN);
  static constexpr int kThreads = 64 * kWaves;
  static constexpr int kCodes = (BM + BN) * kStep;
  static constexpr int kStage = kCodes + 4 * kThreads;  // and a scale of each row and column
  static_assert(BM + BN <= kThreads, "one scale a thread");
};

template <int BM, int BN, int WM, int WN, int OCC, int NS, bool WHOLE, bool ONCE, typename TO>
__global__ __launch_bounds__((TileShape<BM, BN, WM, WN>::kThreads), OCC) void k_matmul_f8_tile(LinearF8Args a, int tiles_m,
                                                                                               int tiles_n, int split_steps,
                                                                                               float* parts) {
  using S = TileShape<BM, BN, WM, WN>;
  constexpr int TM = WM / 16, TN = WN / 16;
  constexpr int NA = BM * 8 / S::kThreads, NB = BN * 8 / S::kThreads;  // 16-byte pieces per thread and step
  constexpr int kRows = S::kThreads / 8;                              // rows that one round of fills covers
  static_assert(kRows % 16 == 0 && NA >= 1 && NB >= 1, "rounds of fills");
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  typedef __attribute__((address_space(3))) void* lds_ptr;

  // neighbouring tiles on one XCD, in bands of 8 tile rows, share operands in its L2
  const int total = tiles_m * tiles_n;
  const uint32_t wg = workgroup<S::kThreads>();
  if (wg >= (uint32_t)total) return;
  const int id = (int)xcd_item(wg, total);
  const int band = id / (8 * tiles_n), in = id - band * 8 * tiles_n;
  const int bm = tiles_m - band * 8 < 8 ? tiles_m - band * 8 : 8;
  const int64_t m0 = (int64_t)(band * 8 + in % bm) * BM, n0 = (int64_t)(in / bm) * BN;

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = (wave % (BM / WM)) * WM, wn = (wave / (BM / WM)) * WN;
  const int K = (int)a.K, K16 = (K + 15) & ~15;

  // fills: thread -> LDS row tid / 8 (+ kRows per round), place tid % 8; and one scale, of row or column tid
  const int frow = tid >> 3;
  const int pa = ((tid & 7) ^ key_a(frow)) * 16, pb = ((tid & 7) ^ key_b<TN>(frow)) * 16;
  Bytes ra[NA], rb[NB];  // of the rounds' first rows on
#pragma unroll
  for (int i = 0; i < NA; ++i) ra[i] = bytes_from(a.A, m0 + i * kRows, a.M, a.lda, K16);
#pragma unroll
  for (int i = 0; i < NB; ++i) rb[i] = bytes_from(a.B, n0 + i * kRows, a.N, a.ldb, K16);

  const int all = (K + kStep - 1) / kStep;
  const int first = (int)blockIdx.z * split_steps;  // this workgroup's steps of the sum
  const int steps = all - first < split_steps ? all - first : split_steps;

  const int oa = frow * (int)a.lda + pa, ob = frow * (int)a.ldb;
  const bool of_a = tid < BM;
  const int64_t sm = m0 + tid < a.M ? m0 + tid : a.M - 1, sn = n0 + tid - BM < a.N ? n0 + tid - BM : a.N - 1;
  const float* scales = of_a ? a.a_scale + first * a.M + sm : a.b_scale + sn / kBlockF8 * all + first;
  const int64_t next_scale = of_a ? a.M : 1;
  // Part c of step t's fills: a round of A's or B's rows, or the scales.  Past the last step they come from beyond the
  // operands: they keep the counts and read nothing.
  constexpr int kParts = NA + NB + 1;
  const auto fill = [&](int stage, int t, int c) {
    const int k = t < steps ? (first + t) * kStep : K;
    char* base = lds + stage * S::kStage;
    if (c < NA) {
      fill16<false>(ra[c], base + wave * 1024 + c * kRows * kStep, k + pa + 16 <= K ? oa + k : (int)0x80000000);
    } else if (c < NA + NB) {
      const int i = c - NA, p = pb ^ ((i * kRows / (4 * TN)) & 3) << 5;  // the key of the round's rows
      fill16<ONCE>(rb[i], base + wave * 1024 + (BM + i * kRows) * kStep, k + p + 16 <= K ? ob + p + k : (int)0x80000000);
    } else {
      __builtin_amdgcn_global_load_lds((__attribute__((address_space(1))) void*)scales, (lds_ptr)(base + S::kCodes + wave * 256), 4, 0, 0);
      if (t + 1 < steps) scales += next_scale;  // (past the last step the last scales again: nothing uses them)
    }
  };
  // fragments: lane -> row lane % 16 of the operand, pieces lane / 16 and lane / 16 + 4
  const int g = lane >> 4, r = lane & 15;
  const int rb_n = 4 * TN * (r >> 2) + (r & 3);
  const int qa = (g ^ key_a(r)) * 16, qb = (g ^ key_b<TN>(rb_n)) * 16;
  const auto read_a = [&](int stage, int j) {
    const char* p = lds + stage * S::kStage + (wm + 16 * j + r) * kStep;
    Operand x;
    x.set(*reinterpret_cast<const i32x4*>(p + qa), *reinterpret_cast<const i32x4*>(p + (qa ^ 64)));
    return x;
  };
  const auto read_b = [&](int stage, int i) {
    const char* p = lds + stage * S::kStage + (BM + wn + rb_n + 4 * i) * kStep;
    Operand w;
    w.set(*reinterpret_cast<const i32x4*>(p + qb), *reinterpret_cast<const i32x4*>(p + (qb ^ 64)));
    return w;
  };
  const auto scale_a = [&](int stage, int j) {
    return *reinterpret_cast<const float*>(lds + stage * S::kStage + S::kCodes + (wm + 16 * j + r) * 4);
  };
  const auto scale_b = [&](int stage) {
    return *reinterpret_cast<const float*>(lds + stage * S::kStage + S::kCodes + (BM + wn) * 4);
  };

  // waits until the oldest fills are in, this wavefront's and then everyone's (`later` parts follow them)
  const auto arrived = [&](auto later) {
    constexpr int n = decltype(later)::value;
    static_assert(n < 64, "vmcnt");
    __builtin_amdgcn_s_waitcnt(0x0F70 | (n & 15) | (n >> 4) << 14);  // vmcnt(n)
    sync_lds();                                                    // (every fragment of the stage that is refilled next is read)
  };

  fl4 acc[TN][TM];
#pragma unroll
  for (int i = 0; i < TN; ++i)
#pragma unroll
    for (int j = 0; j < TM; ++j) acc[i][j] = fl4{0, 0, 0, 0};

  // A product that follows a step's meeting, TN - 1 of them in its last phase and then those of the next step's phases, has
  // kPer parts of the fills after it, so that they do not stop a wavefront for as long as they take to go out together
  // (4096 x 4096 x 40960: 1097 us with all parts after one product, 1081; in four stages 1409 and 1339).
  constexpr int kSlots = TN - 1 + (TM - 1) * TN;
  constexpr int kPer = (4 * kParts + 3 * kSlots - 1) / (3 * kSlots);
  constexpr int kFirst = WHOLE || (TN - 1) * kPer > kParts ? kParts : (TN - 1) * kPer;  // parts in the last phase
  const auto fills = [&](int stage, int t, int slot) {
#pragma unroll
    for (int c = slot * kPer; c < (slot + 1) * kPer && c < kParts; ++c) fill(stage, t, c);
  };
#pragma unroll
  for (int t = 0; t < NS; ++t)
#pragma unroll
    for (int c = 0; c < (t + 1 < NS ? kParts : kFirst); ++c) fill(t, t, c);
  arrived(std::integral_constant<int, (NS - 2) * kParts + kFirst>{});
  int st = 0;
  Operand w[TN], x;
  float s;
  if constexpr (WHOLE) {
    // A step's operands are all read while the products of the step before run, into the other of two sets of registers (tiles
    // of 128 x 128 have not the registers).
    Operand fa[2][TM], fb[2][TN];
    float sc[2][TM];
    const auto read = [&](int stage, int b) {
      const float sb = scale_b(stage);
#pragma unroll
      for (int i = 0; i < TN; ++i) fb[b][i] = read_b(stage, i);
#pragma unroll
      for (int j = 0; j < TM; ++j) {
        fa[b][j] = read_a(stage, j);
        sc[b][j] = scale_a(stage, j) * sb;
      }
    };
    read(0, 0);
    for (int t0 = 0; t0 < steps; t0 += 2) {
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const int t = t0 + b;
        if (t >= steps) break;
        const int next = st + 1 == NS ? 0 : st + 1;
        arrived(std::integral_constant<int, (NS - 2) * kParts>{});
        read(next, b ^ 1);
#pragma unroll
        for (int c = 0; c < kParts; ++c) fill(st, t + NS, c);
        fl4 q[TN][TM];
#pragma unroll
        for (int i = 0; i < TN; ++i)
#pragma unroll
          for (int j = 0; j < TM; ++j) q[i][j] = sums_of(fb[b][i], fa[b][j]);
#pragma unroll
        for (int i = 0; i < TN; ++i)
#pragma unroll
          for (int j = 0; j < TM; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[i][j][e] = __builtin_fmaf(q[i][j][e], sc[b][j], acc[i][j][e]);
        st = next;
      }
    }
  } else {
    // A phase multiplies one operand of A with all of B's, and adds the sums of the phase before while the matrix cores
    // work.  The next operand is read at the phase's beginning.  In a step's last phase the workgroup meets after the first
    // product, and the next step's operands and the fills of the one after it follow, each of B's operands into
    // the registers that a product has just been the last to use.
    x = read_a(0, 0);
#pragma unroll
    for (int i = 0; i < TN; ++i) w[i] = read_b(0, i);
    float sb_now = scale_b(0);
    s = scale_a(0, 0) * sb_now;
    fl4 p[TN];
#pragma unroll
    for (int i = 0; i < TN; ++i) p[i] = fl4{0, 0, 0, 0};
    float s_was = 0.0f;
    const auto product = [&](int i, int before) {
      const fl4 q = sums_of(w[i], x);
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[i][before][e] = __builtin_fmaf(p[i][e], s_was, acc[i][before][e]);
      p[i] = q;
    };
    for (int t = 0; t < steps; ++t) {
      const int next = st + 1 == NS ? 0 : st + 1, prev = st == 0 ? NS - 1 : st - 1;
      Operand y;
      float s_next;
#pragma unroll
      for (int j = 0; j + 1 < TM; ++j) {
        y = read_a(st, j + 1);
        s_next = scale_a(st, j + 1) * sb_now;
#pragma unroll
        for (int i = 0; i < TN; ++i) {
          product(i, j == 0 ? TM - 1 : j - 1);
          fills(prev, t - 1 + NS, TN - 1 + j * TN + i);
        }
        __builtin_amdgcn_sched_group_barrier(0x100, 3, 0);  // LDS read
#pragma unroll
        for (int i = 0; i < TN; ++i) {
          __builtin_amdgcn_sched_group_barrier(0x008, 4, 0);  // MFMA
          __builtin_amdgcn_sched_group_barrier(0x020, kPer, 0);                     // memory read
          __builtin_amdgcn_sched_group_barrier(0x002, 4, 0);                        // VALU
        }
        __builtin_amdgcn_sched_barrier(0);
        x = y;
        s_was = s;
        s = s_next;
      }
#pragma unroll
      for (int i = 0; i < TN; ++i) {
        product(i, TM == 1 ? 0 : TM - 2);
        __builtin_amdgcn_sched_barrier(0);
        if (i == 0) {
          arrived(std::integral_constant<int, (NS - 2) * kParts>{});
          y = read_a(next, 0);
          sb_now = scale_b(next);
          s_next = scale_a(next, 0);
        }
        w[i] = read_b(next, i);
        if (i > 0) fills(st, t + NS, i - 1);
        __builtin_amdgcn_sched_barrier(0);
      }
      x = y;
      s_was = s;
      s = s_next * sb_now;
      st = next;
    }
#pragma unroll
    for (int i = 0; i < TN; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[i][TM - 1][e] = __builtin_fmaf(p[i][e], s_was, acc[i][TM - 1][e]);
  }
  __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0): no fill outlives the workgroup
  if (K % 16 && first + steps == all) {
    const int64_t k = K & ~15;
    const i32x4 none = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < TN; ++i) {
      const int64_t n = n0 + wn + rb_n + 4 * i;
      w[i].set(g == 0 ? piece(a.B + (n < a.N ? n : a.N - 1) * a.ldb + k, K - k) : none, none);
    }
    const int64_t nb0 = n0 + wn < a.N ? n0 + wn : a.N - 1;
    const float sb_last = a.b_scale[nb0 / kBlockF8 * all + all - 1];
#pragma unroll
    for (int j = 0; j < TM; ++j) {
      const int64_t m = m0 + wm + 16 * j + r < a.M ? m0 + wm + 16 * j + r : a.M - 1;
      x.set(g == 0 ? piece(a.A + m * a.lda + k, K - k) : none, none);
      s = a.a_scale[(all - 1) * a.M + m] * sb_last;
#pragma unroll
      for (int i = 0; i < TN; ++i) {
        const fl4 q = sums_of(w[i], x);
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[i][j][e] = __builtin_fmaf(q[e], s, acc[i][j][e]);
      }
    }
  }

  // results: lane -> row wm + 16 j + r, columns wn + 4 TN g + 4 i + e
  const int64_t n = n0 + wn + 4 * TN * g;
  if (parts) {  // a part of the sum, for k_matmul_f8_join
    float* o = parts + (int64_t)blockIdx.z * a.M * a.N;
#pragma unroll
    for (int j = 0; j < TM; ++j) {
      const int64_t m = m0 + wm + 16 * j + r;
      if (m >= a.M) continue;
#pragma unroll
      for (int i = 0; i < TN; ++i) {
        if (n + 4 * i + 4 <= a.N && (a.N & 3) == 0) {
          *reinterpret_cast<fl4*>(o + m * a.N + n + 4 * i) = acc[i][j];
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (n + 4 * i + e < a.N) o[m * a.N + n + 4 * i + e] = acc[i][j][e];
        }
      }
    }
    return;
  }
  float bias[TN][4];
#pragma unroll
  for (int i = 0; i < TN; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int64_t nn = n + 4 * i + e;
      bias[i][e] = a.bias ? a.bias[nn < a.N ? nn : a.N - 1] : 0.0f;
    }
  // Results go out through the wavefront's own part of LDS (the stages are done with), so that a store covers whole lines.
  constexpr int V = 16 / sizeof(TO), kPieces = WN / V;  // values of a piece, pieces of a row
  constexpr int kMine = NS * S::kStage / S::kWaves / (16 * kPieces * 16);  // m-tiles that the part holds
  constexpr int G = kMine >= TM ? TM : kMine >= TM / 2 ? TM / 2 : TM / 4;
  static_assert(G >= 1 && TM % G == 0, "LDS of the results");
  typedef TO Piece __attribute__((ext_vector_type(16 / sizeof(TO))));
  char* mine = lds + wave * (G * 16 * kPieces * 16);
  const bool wide = ((reinterpret_cast<uintptr_t>(a.out) | (uintptr_t)(a.ldo * sizeof(TO))) & 15) == 0;
  __syncthreads();
#pragma unroll
  for (int j0 = 0; j0 < TM; j0 += G) {
#pragma unroll
    for (int j = j0; j < j0 + G; ++j) {
      const int row = 16 * (j - j0) + r;
#pragma unroll
      for (int q = 0; q < 4 * TN / V; ++q) {
        Piece w8;
#pragma unroll
        for (int e = 0; e < V; ++e) {
          const int c = q * V + e;
          w8[e] = (TO)rounded(acc[c / 4][j][c % 4] + bias[c / 4][c % 4]);
        }
        const int at = 4 * TN / V * g + q;
        *reinterpret_cast<Piece*>(mine + (row * kPieces + (at ^ ((row >> 1) & (kPieces - 1)))) * 16) = w8;
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    TO* o = static_cast<TO*>(a.out) + (m0 + wm + 16 * j0) * a.ldo + n0 + wn;
    const int64_t rows_left = a.M - (m0 + wm + 16 * j0), left = a.N - (n0 + wn);
    if (wide && left >= WN) {
#pragma unroll
      for (int q = 0; q < G * 16 * kPieces / 64; ++q) {
        const int y = q * 64 + lane, row = y / kPieces, at = y % kPieces;
        const Piece w8 = *reinterpret_cast<const Piece*>(mine + (row * kPieces + (at ^ ((row >> 1) & (kPieces - 1)))) * 16);
        if (row < rows_left) *reinterpret_cast<Piece*>(o + row * a.ldo + at * V) = w8;
      }
    } else {  // rows that do not lie on 16 bytes, or the last columns
#pragma unroll 4
      for (int q = 0; q < G * 16 * WN / 64; ++q) {
        const int y = q * 64 + lane, row = y / WN, col = y % WN;
        const char* c = mine + (row * kPieces + ((col / V) ^ ((row >> 1) & (kPieces - 1)))) * 16 + col % V * sizeof(TO);
        if (row < rows_left && col < left) o[row * a.ldo + col] = *reinterpret_cast<const TO*>(c);
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  }
}

// The parts of split sums together, with the epilogue; four columns a thread.  In the order of the parts: the same bits
// every time.  About 2 us, of launch and latency.
template <typename TO>
__global__ __launch_bounds__(256) void k_matmul_f8_join(LinearF8Args a, const float* __restrict__ parts, int n_parts) {
  const int64_t quads = (a.N + 3) / 4;
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= quads * a.M) return;
  const int64_t m = i / quads, n = (i - m * quads) * 4;
  float sum[4] = {0, 0, 0, 0};
  for (int p = 0; p < n_parts; ++p) {
    const float* q = parts + ((int64_t)p * a.M + m) * a.N + n;
    if ((a.N & 3) == 0) {
      const fl4 v = *reinterpret_cast<const fl4*>(q);
#pragma unroll
      for (int e = 0; e < 4; ++e) sum[e] += v[e];
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) sum[e] += n + e < a.N ? q[e] : 0;
    }
  }
  TO* o = static_cast<TO*>(a.out) + m * a.ldo;
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (n + e < a.N) o[n + e] = (TO)rounded(sum[e] + (a.bias ? a.bias[n + e] : 0.0f));
}

template <int BM, int BN, int WM, int WN, int OCC, int NS, bool WHOLE, bool ONCE, typename TO>
hipError_t launch_tile(const LinearF8Args& a, int split, void* ws, hipStream_t st) {
  using S = TileShape<BM, BN, WM, WN>;
  const auto k = k_matmul_f8_tile<BM, BN, WM, WN, OCC, NS, WHOLE, ONCE, TO>;
  const size_t lds = NS * S::kStage;
  if (lds > 65536) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(k), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return e;
  }
  const int64_t tm = (a.M + BM - 1) / BM, tn = (a.N + BN - 1) / BN;
  if (tm * tn > 0x7FFFFFFF) return hipErrorInvalidValue;  // (8 TB of results)
  const int all = (int)((a.K + kStep - 1) / kStep), per = (all + split - 1) / split;
  split = (all + per - 1) / per;
  float* parts = split > 1 ? static_cast<float*>(ws) : nullptr;
  dim3 grid = grid_of<S::kThreads>(tm * tn);
  grid.z = (unsigned)split;
  hipLaunchKernelGGL(k, grid, dim3(S::kThreads), lds, st, a, (int)tm, (int)tn, per, parts);
  if (parts) {
    const int64_t quads = a.M * ((a.N + 3) / 4);
    hipLaunchKernelGGL((k_matmul_f8_join<TO>), dim3((unsigned)((quads + 255) / 256)), dim3(256), 0, st, a, parts, split);
  }
  return hipGetLastError();
}

// Bytes between rows of codes in LDS: whole blocks, and 16 more so that rows start in different banks.
int linear_rows_pitch(int64_t K) { return (int)((K + kBlockF8 - 1) / kBlockF8 * kBlockF8 + 16); }
constexpr int kLinearRowsLds = 53248;  // at most, where linear_f8_fused() says so (16 x 2560: 42496, 2 x 20480: 51232)
size_t linear_rows_lds(int64_t M, int64_t K) {
  return (size_t)M * linear_rows_pitch(K) + (size_t)((K + kBlockF8 - 1) / kBlockF8) * 64;
}

// Weights read once that fill a good part of the last cache go past it (64 x 27648 x 5120: 36.8, 33.4 past it; 8 x 27648 x
// 5120 33.3 and 31.4; 16 x 13824 x 5120 22.8 and 22.0; 48 x 20000 x 4096 28.0 and 27.4; 1 x 8192 x 8192 18.9 and 18.2; in the
// caches 64 x 27648 x 5120 32.5 and 33.3).
bool weights_once(int64_t M, int64_t N, int64_t K) { return M <= 64 && N * K >= (int64_t)1 << 26; }

template <int W, int R, typename TO>
hipError_t launch_rows(const LinearF8Args& a, hipStream_t st) {
  auto k = k_matmul_f8_rows<W, R, false, TO>;
  if constexpr (R == 1)  // (more rows take smaller weights only)
    if (weights_once(a.M, a.N, a.K)) k = k_matmul_f8_rows<W, R, true, TO>;
  hipLaunchKernelGGL(k, dim3((unsigned)((a.N + 15) / 16)), dim3(64 * W), 0, st, a);
  return hipGetLastError();
}

template <int W, typename T, typename TO>
hipError_t launch_linear_rows(const LinearF8Args& a, const void* X, int64_t ldx, hipStream_t st) {
  const auto k = weights_once(a.M, a.N, a.K) ? k_linear_f8_rows<W, true, T, TO> : k_linear_f8_rows<W, false, T, TO>;
  const size_t lds = linear_rows_lds(a.M, a.K);
  if (lds > kLinearRowsLds) return hipErrorInvalidValue;
  if (lds > 32768) {  // (beside the sums of 16 wavefronts; the same limit in every call: another thread's may come in between)
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(k), hipFuncAttributeMaxDynamicSharedMemorySize, kLinearRowsLds);
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL(k, dim3((unsigned)((a.N + 15) / 16)), dim3(64 * W), lds, st, a, static_cast<const T*>(X), ldx, linear_rows_pitch(a.K));
  return hipGetLastError();
}
template <int W, typename T>
hipError_t launch_linear_rows_w(const LinearF8Args& a, const void* X, int64_t ldx, hipStream_t st) {
  if (a.out_dtype == AWSRC_DTYPE_F32) return launch_linear_rows<W, T, float>(a, X, ldx, st);
  if (a.out_dtype == AWSRC_DTYPE_BF16) return launch_linear_rows<W, T, __bf16>(a, X, ldx, st);
  return launch_linear_rows<W, T, _Float16>(a, X, ldx, st);
}
template <typename T>
hipError_t launch_linear_rows_t(const LinearF8Args& a, const void* X, int64_t ldx, hipStream_t st) {
  // sixteen wavefronts where the workgroups leave CUs idle (with eight and sixteen: 1 x 2048 x 11008 10.7 and 10.2; 3 x 2048 x 11008
  // 13.3 and 12.3; 16 x 2048 x 2048 7.7 and 6.7; 8 x 4096 x 2048 6.2 and 5.8; 1 x 2560 x 2048 4.3 and 4.3; 1 x 5120 x 5120 10.0
  // and 11.5; 9 x 11008 x 2048 12.3 and 15.4)
  return a.N <= 4096 && (a.M >= 4 || a.K >= 8192) ? launch_linear_rows_w<16, T>(a, X, ldx, st)
                                                  : launch_linear_rows_w<8, T>(a, X, ldx, st);
}

// Which kernel takes a product, and over how many parts of the sum.  Times below are in us, into bf16, of calls on
// weights that are not in the caches; into fp32 they are within a tenth.
enum Path { kRows, kTile32, kTile64, kTile64Wide, kTile128Deep, kTile128 };
struct Choice {
  Path path;
  int split;
};
Choice choose(int64_t M, int64_t N, int64_t K) {
  const auto tiles = [&](int64_t bm, int64_t bn) { return ((M + bm - 1) / bm) * ((N + bn - 1) / bn); };
  // Up to 16 rows: 16 columns a workgroup, up to about three of them a CU (16 x 2048 x 11008: 12.0, tiles 14.5 with their
  // sums split; 16 x 11008 x 2048: 9.6 and 11.5; 16 x 13824 x 5120: 23.1 and 22.0; 8 x 27648 x 5120: 38.1 and 31.4).
  if (M <= 16 && N < 12288) return {kRows, 1};
  // Up to 32 rows of weights that are not too large, nor with too many columns (32 x 4096 x 4096: 9.1 and 12.3; 24 x 5120 x 5120:
  // 16.3 and 16.2; 32 x 8192 x 8192: 25.3 and 23.1; 24 x 8192 x 2400: 12.0 and 11.8; 24 x 11008 x 1024: 9.0 and 7.8; 24 x 27648 x
  // 512: 18.6 and 8.3).
  if (M > 16 && M <= 32 && N * K <= 20000000 && N <= 8192) return {kRows, 1};
  const int64_t wide = tiles(64, 128), t128 = tiles(128, 128);
  // 64 x 128 tiles where a CU has one at most, and 64 x 64 ones would not all have a CU: 64 x 27648 x 5120: 64 x 64 tiles 38.5,
  // 33.4; 48 x 20000 x 4096: 28.5 and 27.4; 256 x 8192 x 8192: 54.7 and 49.2; 1000 x 2048 x 11008: 70 and 63.
  if (M > 32 && wide > 128 && (wide <= 256 || M <= 64)) return {kTile64Wide, 1};
  // 128 x 128 tiles with four stages where a CU has one of them (128 x 27648 x 5120: 51.6, 64 x 128 tiles 57.3, with two stages
  // 66.9; 512 x 5120 x 5120: 48.5, 47.4 and 59.7; 200 x 11008 x 2048: 23.3, 22.7 and 27.5), 64 x 128 ones where a CU has two of
  // those (320 x 11008 x 5120: 49.2, 128 x 128 tiles 70.3).
  if (M > 64 && wide > 256 && t128 <= 256) return {kTile128Deep, 1};
  if (M > 64 && wide > 256 && wide <= 512) return {kTile64Wide, 1};
  // 128 x 128 tiles, two workgroups a CU (4096 x 5120 x 5120: 193, 64 x 128 tiles 231; 1000 x 11008 x 2048: 55 and 61).
  if (M > 64 && wide > 512) return {kTile128, 1};
  const Path path = M > 32 ? kTile64 : kTile32;
  // Few tiles under a long sum: as many parts as cost least, joined by a second launch.  A step costs 0.48 us;
  // the join 2.1, 0.3 more a part and what the parts' bytes take (64 x 2048 x 11008: 41 whole, 15.7 in 8 parts, 19.5 in 16; 256
  // x 1024 x 4096: 17.7, 12.5 in 4, 15.1 in 8; 128 x 2048 x 2048: 10.8 whole, 10.9 in 2).  And half of the 3 that a launch
  // costs the host where it is not replayed from a graph.
  const int64_t t = path == kTile64 ? tiles(64, 64) : tiles(32, 64), steps = (K + kStep - 1) / kStep;
  const double step = 0.48, bytes = 1.8e-6 * (double)M * (double)N;
  Choice best = {path, 1};
  double least = step * (double)steps;
  for (int s = 2; s <= 16 && s * t <= 256; ++s) {
    const double us = 2.1 + 1.5 + 0.3 * s + step * (double)((steps + s - 1) / s) + bytes * s;
    if (us < least) {
      least = us;
      best.split = s;
    }
  }
  return best;
}

template <typename TO>
hipError_t launch(const LinearF8Args& a, void* ws, hipStream_t st) {
  const Choice c = choose(a.M, a.N, a.K);
  const bool once = weights_once(a.M, a.N, a.K);
  switch (c.path) {
    case kRows: return a.M <= 16 ? launch_rows<8, 1, TO>(a, st) : launch_rows<8, 2, TO>(a, st);
    case kTile32:
      return once ? launch_tile<32, 64, 32, 32, 2, 4, true, true, TO>(a, c.split, ws, st)
                  : launch_tile<32, 64, 32, 32, 2, 4, true, false, TO>(a, c.split, ws, st);
    case kTile64:
      return once ? launch_tile<64, 64, 32, 32, 2, 4, true, true, TO>(a, c.split, ws, st)
                  : launch_tile<64, 64, 32, 32, 2, 4, true, false, TO>(a, c.split, ws, st);
    case kTile64Wide:
      return once ? launch_tile<64, 128, 32, 64, 2, 3, true, true, TO>(a, 1, ws, st)
                  : launch_tile<64, 128, 32, 64, 2, 3, true, false, TO>(a, 1, ws, st);
    case kTile128Deep: return launch_tile<128, 128, 64, 64, 2, 4, false, false, TO>(a, 1, ws, st);
    default: return launch_tile<128, 128, 64, 64, 2, 2, false, false, TO>(a, 1, ws, st);
  }
}

}  // namespace

size_t matmul_f8_ws_bytes(int64_t M, int64_t N, int64_t K) {
  const int split = choose(M, N, K).split;
  return split > 1 ? (size_t)split * (size_t)M * (size_t)N * 4 : 0;
}

hipError_t launch_matmul_f8(const LinearF8Args& a, void* ws, hipStream_t st) {
  if (a.out_dtype == AWSRC_DTYPE_F32) return launch<float>(a, ws, st);
  if (a.out_dtype == AWSRC_DTYPE_BF16) return launch<__bf16>(a, ws, st);
  return launch<_Float16>(a, ws, st);
}

bool linear_f8_fused(int64_t M, int64_t N, int64_t K) {
  // Where quantizing over and over costs a workgroup less than a launch, or little more: one that is not replayed from a graph
  // costs the host 3.  On the GPU, in us, fused and in two launches: 1 x 2560 x 2048 4.3 and 6.4; 1 x 11008 x 2048 8.8 and 12.2; 1 x
  // 27648 x 5120 30.4 and 35.8; 1 x 5120 x 27648 35.2 and 46.1; 2 x 5120 x 5120 11.0 and 14.2; 4 x 5120 x 5120 13.1 and 14.3; 8 x
  // 11008 x 2048 11.9 and 12.2; 16 x 2048 x 2560 7.9 and 7.2; 8 x 5120 x 5120 16.9 and 14.7; 16 x 11008 x 2048 16.7 and 12.3; 16 x
  // 2048 x 4096 11.2 and 8.3.
  if (M == 1) return K <= 32768 && N <= (int64_t)1 << 26;  // (2^31 threads of a launch)
  return M <= 16 && N < 12288 && M * K <= (N <= 4096 ? 40960 : 20480);
}

hipError_t launch_linear_f8_fused(const LinearF8Args& a, const void* X, int x_dtype, int64_t ldx, hipStream_t st) {
  if (x_dtype == AWSRC_DTYPE_F32) return launch_linear_rows_t<float>(a, X, ldx, st);
  if (x_dtype == AWSRC_DTYPE_BF16) return launch_linear_rows_t<__bf16>(a, X, ldx, st);
  return launch_linear_rows_t<_Float16>(a, X, ldx, st);
}

}  // namespace awsrc
