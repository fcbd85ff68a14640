// Drafted tokens against the target's probabilities.
//
// Only one row of p (and of q) is read whole for each sequence: the one that
// its next token is drawn from, known from single entries of the rows before it.
// Where one CU reads that row quickly enough, one workgroup a sequence does it all.
// Longer rows take two launches: sums of the weights over pieces of the row, every
// wavefront finding the row by itself; then one workgroup a sequence finds the piece in
// which the running sum passes its mark, and the token in it.  Sums in fp64: a
// product u q of fp32 numbers is exact there, and the order of adding moves a border
// between tokens by 1e-16 of the whole.
//
// Bound by the rows' bytes for a batch, for one sequence by memory's latency: offsets,
// tokens, their probabilities, the row and a piece of it again wait for one another.
// One sequence of four drafts and 32768 tokens in fp32 6.8 us; 64 of 131072 with their
// drafts' probabilities 9.4 (67 MB, 7 TB/s: some of it from the last level of cache) + 5.3.
#include "serve_internal.h"

namespace awsrc {

namespace {

constexpr int kThreads = 256;
constexpr int kPiece = 2048;  // tokens of a piece of a row, 8 of a thread in the second launch

struct Rows {
  int64_t begin, n;  // of a sequence
};
__device__ __forceinline__ Rows rows_of(const VerifyArgs& a, int s) {
  int64_t r0 = a.cu[s], r1 = a.cu[s + 1];
  r0 = r0 < 0 ? 0 : r0 < a.n_rows ? r0 : a.n_rows;
  r1 = r1 < r0 ? r0 : r1 < a.n_rows ? r1 : a.n_rows;
  return {r0, r1 - r0};
}

// The first row (counted from the sequence's first) whose draft is refused, or the last one; by one wavefront.
template <typename T>
__device__ __forceinline__ int64_t place_of(const VerifyArgs& a, Rows rows) {
  const int lane = threadIdx.x & 63;
  for (int64_t base = 0; base < rows.n - 1; base += 64) {
    const int64_t i = base + lane, r = rows.begin + i;
    bool refused = false;
    if (i < rows.n - 1) {
      const int64_t x = a.tokens[r + 1];
      refused = true;
      if (x >= 0 && x < a.vocab) {
        const double p = (double)to_f32(static_cast<const T*>(a.p)[r * a.ldp + x]);
        const double q = a.q ? (double)to_f32(static_cast<const T*>(a.q)[r * a.ldq + x]) : 1.0;
        refused = !((double)a.u[r] * q < p);
      }
    }
    const uint64_t any = __ballot(refused);
    if (any) return base + __builtin_ctzll(any);
  }
  return rows.n - 1;
}

// The weights that a sequence's token is drawn from.
template <typename T>
struct Weights {
  const T *p, *q;  // q NULL where only p counts
  int64_t vocab, less;  // less: a token that counts one less, -1 for none
  __device__ __forceinline__ Weights(const VerifyArgs& a, Rows rows, int64_t place) : vocab(a.vocab) {
    const int64_t r = rows.begin + place;
    const bool cut = place < rows.n - 1;
    p = static_cast<const T*>(a.p) + r * a.ldp;
    q = a.q && cut ? static_cast<const T*>(a.q) + r * a.ldq : nullptr;
    less = !a.q && cut ? a.tokens[r + 1] : -1;
  }
  __device__ __forceinline__ bool plain() const { return !q && less < 0; }
  // p's own probabilities from here on
  __device__ __forceinline__ void make_plain() {
    q = nullptr;
    less = -1;
  }
  __device__ __forceinline__ void load(int64_t i, float (&x)[8], float (&y)[8]) const {
    load8_any(p + i, vocab - i, x);
    if (q) load8_any(q + i, vocab - i, y);
  }
  // the weight of token i of the values loaded: 0 where one is not finite or the difference not positive, exact otherwise
  // but for the rounding of a difference to 53 bits
  __device__ __forceinline__ double of(int64_t i, float x, float y) const {
    constexpr float inf = __builtin_inff();
    const float l = q ? y : i == less ? 1.0f : 0.0f;
    return x > l && x < inf && l > -inf ? (double)x - (double)l : 0.0;
  }
};

// 16 bytes of a row from any element on.
template <typename T>
struct Vec {
  static constexpr int n = 16 / sizeof(T);
  typedef T type __attribute__((ext_vector_type(16 / sizeof(T)), aligned(sizeof(T))));
};

// The sum of a piece's weights, by one wavefront, whose eight or sixteen loads a lane and row are on their way together; in
// lane 63.
//
// Weights that are not finite show in the sum, which is then made again value by value: a maximum with 0 is all that
// a weight costs besides its conversion and its addition (200 rows of 100003 in bf16 12.7 us, 18.0 with every value compared).
template <typename T>
__device__ __forceinline__ double sum_of_piece(const Weights<T>& weights, int64_t piece) {
  typedef typename Vec<T>::type V;
  constexpr int n = Vec<T>::n, kLoads = kPiece / (64 * n);
  const int lane = threadIdx.x & 63;
  const int64_t begin = piece * kPiece, end = begin + kPiece;
  double w = __builtin_inf();
  if (end <= weights.vocab && !(weights.less >= begin && weights.less < end)) {
    const T* p = weights.p + begin + lane * n;
    V x[kLoads];
#pragma unroll
    for (int j = 0; j < kLoads; ++j) x[j] = *reinterpret_cast<const V*>(p + j * 64 * n);
    w = 0.0;
    if (weights.q) {
      const T* q = weights.q + begin + lane * n;
      V y[kLoads];
#pragma unroll
      for (int j = 0; j < kLoads; ++j) y[j] = *reinterpret_cast<const V*>(q + j * 64 * n);
#pragma unroll
      for (int j = 0; j < kLoads; ++j)
#pragma unroll
        for (int e = 0; e < n; ++e) w += __builtin_fmax((double)to_f32((T)x[j][e]) - (double)to_f32((T)y[j][e]), 0.0);
    } else {
#pragma unroll
      for (int j = 0; j < kLoads; ++j)
#pragma unroll
        for (int e = 0; e < n; ++e) w += (double)__builtin_fmaxf(to_f32((T)x[j][e]), 0.0f);
    }
    w = scan_wave(w);
  }
  if (!(of_lane(w, 63) < __builtin_inf())) {  // the row ends in here, the draft lies here, or a value is not finite
    w = 0.0;
    float x[kPiece / 512][8], y[kPiece / 512][8];
#pragma unroll
    for (int j = 0; j < kPiece / 512; ++j) weights.load(begin + (j * 64 + lane) * 8, x[j], y[j]);
#pragma unroll
    for (int j = 0; j < kPiece / 512; ++j)
#pragma unroll
      for (int e = 0; e < 8; ++e) w += weights.of(begin + (j * 64 + lane) * 8 + e, x[j][e], y[j][e]);
    w = scan_wave(w);
  }
  return w;
}

// A wavefront takes two pieces of 16-bit values, one of fp32 ones.
template <typename T>
constexpr int kPerWave = sizeof(T) == 2 ? 2 : 1;

template <typename T>
__global__ __launch_bounds__(kThreads) void k_verify_sums(VerifyArgs a, int pieces, uint32_t groups, int64_t n_wg, double* sums,
                                                          int32_t* places) {
  const uint32_t wg = workgroup<kThreads>();
  if (wg >= n_wg) return;
  const int s = (int)(wg / groups), first = ((int)(wg % groups) * (kThreads / 64) + (threadIdx.x >> 6)) * kPerWave<T>;
  const Rows rows = rows_of(a, s);
  if (rows.n == 0 || first >= pieces) return;
  const int64_t place = place_of<T>(a, rows);
  const Weights<T> weights(a, rows, place);
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int k = 0; k < kPerWave<T>; ++k) {
    if (first + k >= pieces) break;
    const double w = sum_of_piece(weights, first + k);
    if (lane == 63) sums[(int64_t)s * pieces + first + k] = w;
  }
  if (first == 0 && lane == 0) places[s] = (int32_t)place;
}

// Rows that are not too long: one workgroup a sequence does it all, without a workspace.  Every wavefront finds the row and sums
// pieces of it; the first one then draws, its lanes holding 32 tokens side by side.
constexpr int kAlone = 64;  // pieces at most, one a lane
constexpr int kAloneWaves = 16;

template <typename T>
__global__ __launch_bounds__(64 * kAloneWaves) void k_verify_alone(VerifyArgs a, int pieces) {
  __shared__ double sums[64];
  const uint32_t s = workgroup<64 * kAloneWaves>();
  if (s >= (uint32_t)a.n_seq) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const Rows rows = rows_of(a, (int)s);
  int64_t place = -1, token = -1;
  if (rows.n > 0) {
    place = place_of<T>(a, rows);
    const float u = a.u[rows.begin + rows.n - 1];
    Weights<T> weights(a, rows, place);
    if (tid < 64) sums[tid] = 0.0;
    double upto, all;
    for (;;) {
      __syncthreads();
      for (int c = wave; c < pieces; c += kAloneWaves) {
        const double w = sum_of_piece(weights, c);
        if (lane == 63) sums[c] = w;
      }
      __syncthreads();
      upto = scan_wave(sums[lane]);
      all = of_lane(upto, 63);
      if (all > 0.0 || weights.plain()) break;
      weights.make_plain();  // nothing of p lies above q: p itself
    }
    if (all > 0.0 && wave == 0) {
      const double mark = (double)u * all;
      const uint64_t passes = __ballot(sums[lane] > 0.0 && upto > mark), counts = __ballot(sums[lane] > 0.0);
      const int piece = passes ? (int)__builtin_ctzll(passes) : 63 - (int)__builtin_clzll(counts);
      const double before = of_lane(upto, piece) - sums[piece];
      const int64_t at = (int64_t)piece * kPiece + lane * (kPiece / 64);
      float x[kPiece / 512][8], y[kPiece / 512][8];
#pragma unroll
      for (int j = 0; j < kPiece / 512; ++j) weights.load(at + j * 8, x[j], y[j]);
      double sum = 0.0;
#pragma unroll
      for (int j = 0; j < kPiece / 512; ++j)
#pragma unroll
        for (int e = 0; e < 8; ++e) sum += weights.of(at + j * 8 + e, x[j][e], y[j][e]);
      double run = before + (scan_wave(sum) - sum);
      int first = -1, last = -1;
#pragma unroll
      for (int j = 0; j < kPiece / 512; ++j)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const double w = weights.of(at + j * 8 + e, x[j][e], y[j][e]);
          run += w;
          if (w > 0.0) {
            if (first < 0 && run > mark) first = j * 8 + e;
            last = j * 8 + e;
          }
        }
      const uint64_t here = __ballot(first >= 0), some = __ballot(last >= 0);
      const int l = here ? (int)__builtin_ctzll(here) : 63 - (int)__builtin_clzll(some);
      token = (int64_t)piece * kPiece + l * (kPiece / 64) + __shfl(here ? first : last, l, 64);
    }
  }
  if (wave) return;
  for (int64_t i = lane; i < rows.n; i += 64)
    a.tokens_out[rows.begin + i] = i < place ? a.tokens[rows.begin + i + 1] : i == place ? (int32_t)token : -1;
  if (lane == 0) {
    a.n_out[s] = (int32_t)(place + 1);
    if (a.keep) a.keep[s] = (int32_t)(a.kv_len[s] - rows.n + place + 1);
  }
}

__device__ __forceinline__ double scan(double x, double (*wave_sums)[kThreads / 64], double& total) {
  double v[1] = {x}, t[1];
  scan_workgroup<kThreads / 64, 1>(v, t, wave_sums);
  total = t[0];
  return v[0];
}

// The first thread whose running sum passes the mark, or else the last one that counts; one LDS operation a wavefront.
struct Found {
  int first, last;
};
__device__ __forceinline__ void find(Found* f, bool passes, bool counts) {
  const int wave = threadIdx.x >> 6;
  const uint64_t p = __ballot(passes), c = __ballot(counts);
  if ((threadIdx.x & 63) == 0) {
    if (p) atomicMin(&f->first, 64 * wave + (int)__builtin_ctzll(p));
    if (c) atomicMax(&f->last, 64 * wave + 63 - (int)__builtin_clzll(c));
  }
}

template <typename T>
__global__ __launch_bounds__(kThreads) void k_verify_draw(VerifyArgs a, int pieces, double* sums, const int32_t* places) {
  __shared__ double wave_sums[3][kThreads / 64];
  __shared__ Found found[2];
  __shared__ double s_base;
  __shared__ int s_token;
  const uint32_t s = workgroup<kThreads>();
  if (s >= (uint32_t)a.n_seq) return;
  const int tid = threadIdx.x;
  const Rows rows = rows_of(a, (int)s);
  int64_t place = -1, token = -1;
  if (rows.n > 0) {
    place = places[s];
    const float u = a.u[rows.begin + rows.n - 1];
    Weights<T> weights(a, rows, place);
    sums += (int64_t)s * pieces;
    float x[8], y[8];
    if (tid < 2) found[tid] = {0x7FFFFFFF, -1};
    if (tid == 0) s_token = -1;
    double all = 0.0;
    for (int c = tid; c < pieces; c += kThreads) all += sums[c];
    scan(all, &wave_sums[0], all);
    if (!(all > 0.0) && !weights.plain()) {  // nothing of p lies above q: p's own sums, piece by piece
      weights.make_plain();
      for (int c = 0; c < pieces; ++c) {
        const int64_t at = (int64_t)c * kPiece + tid * 8;
        double w = 0.0, total;
        weights.load(at, x, y);
#pragma unroll
        for (int e = 0; e < 8; ++e) w += weights.of(at + e, x[e], y[e]);
        __syncthreads();
        scan(w, &wave_sums[0], total);
        all += total;
        if (tid == 0) sums[c] = total;
      }
      __threadfence_block();
      __syncthreads();
    }
    if (all > 0.0) {
      const double mark = (double)u * all;
      // the piece in which the running sum passes the mark
      double before = 0.0;
      int piece = -1;
      for (int c0 = 0; c0 < pieces; c0 += kThreads) {
        const int c = c0 + tid;
        const double w = c < pieces ? sums[c] : 0.0;
        double total;
        const double upto = before + scan(w, &wave_sums[1], total);
        find(&found[0], w > 0.0 && upto > mark, w > 0.0);
        __syncthreads();
        const bool here = found[0].first != 0x7FFFFFFF;
        if (here || found[0].last >= 0) {
          const int at = here ? found[0].first : found[0].last;
          piece = c0 + at;
          if (tid == at) s_base = upto - w;
        }
        __syncthreads();
        if (here) break;
        if (tid == 0) found[0] = {0x7FFFFFFF, -1};
        before += total;
        __syncthreads();
      }
      // the token in it
      before = s_base;
      const int64_t at = (int64_t)piece * kPiece + tid * 8;
      double w[8], sum = 0.0, total;
      weights.load(at, x, y);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        w[e] = weights.of(at + e, x[e], y[e]);
        sum += w[e];
      }
      double run = before + (scan(sum, &wave_sums[2], total) - sum);
      int first = -1, last = -1;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        run += w[e];
        if (w[e] > 0.0) {
          if (first < 0 && run > mark) first = e;
          last = e;
        }
      }
      find(&found[1], first >= 0, last >= 0);
      __syncthreads();
      const bool here = found[1].first != 0x7FFFFFFF;
      if (tid == (here ? found[1].first : found[1].last)) s_token = (int)(at + (here ? first : last));
      __syncthreads();
      token = s_token;
    }
  }
  if (tid >= 64) return;  // (one wavefront: tokens_out may be tokens)
  for (int64_t i = tid; i < rows.n; i += 64)
    a.tokens_out[rows.begin + i] = i < place ? a.tokens[rows.begin + i + 1] : i == place ? (int32_t)token : -1;
  if (tid == 0) {
    a.n_out[s] = (int32_t)(place + 1);
    if (a.keep) a.keep[s] = (int32_t)(a.kv_len[s] - rows.n + place + 1);
  }
}

template <typename T>
constexpr int kPieces = kPerWave<T> * kThreads / 64;  // of a workgroup of the first launch

int64_t pieces_of(int64_t vocab) { return (vocab + kPiece - 1) / kPiece; }
// A CU reads 131072 probabilities in about as long as two launches take over the whole machine, and a launch less saves the
// host 3 us.  64 sequences of 65536 tokens in fp32 with their drafts' probabilities: 10.7 us, of 65537 in two launches 10.9; 200:
// 16.9 and 17.9; of 131072 in bf16 without them 64: 12.5 and 11.5, 200: 16.3 and 19.8.  A second round of the machine, 300 of
// 65536 in fp32: 25.3 alone and 21.3 in two.
bool verify_alone(int n_seq, int64_t vocab, bool with_q) {
  return pieces_of(vocab) <= kAlone && vocab * (with_q ? 2 : 1) * ((n_seq + 255) / 256) <= kAlone * kPiece;
}

template <typename T>
hipError_t launch(const VerifyArgs& a, void* ws, hipStream_t st) {
  if (verify_alone(a.n_seq, a.vocab, a.q != nullptr)) {
    hipLaunchKernelGGL((k_verify_alone<T>), grid_of<64 * kAloneWaves>(a.n_seq), dim3(64 * kAloneWaves), 0, st, a, (int)pieces_of(a.vocab));
    return hipGetLastError();
  }
  const int64_t pieces = pieces_of(a.vocab), groups = (pieces + kPieces<T> - 1) / kPieces<T>, n = groups * a.n_seq;
  if (n >= (int64_t)1 << 31) return hipErrorInvalidValue;
  double* sums = static_cast<double*>(ws);
  int32_t* places = reinterpret_cast<int32_t*>(sums + pieces * a.n_seq);
  hipLaunchKernelGGL((k_verify_sums<T>), grid_of<kThreads>(n), dim3(kThreads), 0, st, a, (int)pieces, (uint32_t)groups, n, sums, places);
  hipLaunchKernelGGL((k_verify_draw<T>), grid_of<kThreads>(a.n_seq), dim3(kThreads), 0, st, a, (int)pieces, sums, places);
  return hipGetLastError();
}

}  // namespace

// (as for drafts with probabilities of their own, which a query does not know of)
size_t verify_ws_bytes(int n_seq, int64_t vocab) {
  return verify_alone(n_seq, vocab, true) ? 0 : (size_t)n_seq * (pieces_of(vocab) * sizeof(double) + 4);
}

hipError_t launch_verify(const VerifyArgs& a, void* ws, hipStream_t st) {
  if (a.dtype == AWSRC_DTYPE_F32) return launch<float>(a, ws, st);
  if (a.dtype == AWSRC_DTYPE_BF16) return launch<__bf16>(a, ws, st);
  return launch<_Float16>(a, ws, st);
}

}  // namespace awsrc
