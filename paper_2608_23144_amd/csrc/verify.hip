// Drafted tokens against the target's probabilities.
//
// Only one row of p (and of q) is read whole for each sequence: the one that
// its next token is drawn from, known from single entries of the rows before it.  Two
// launches: sums of the weights over pieces of that row, every workgroup finding
// the row by itself; then one workgroup a sequence finds the piece in which the running
// sum passes its mark, and the token in it.  Sums in fp64: a product u q of fp32
// numbers is exact there, and the order of adding moves a border between tokens
// by 1e-16 of the whole.
#include "serve_internal.h"

namespace awsrc {

namespace {

constexpr int kThreads = 256;
template <typename T>
struct Vec {
  static constexpr int n = 16 / sizeof(T);
  typedef T type __attribute__((ext_vector_type(16 / sizeof(T)), aligned(sizeof(T))));
};
constexpr int kPiece = 8192;  // tokens of a workgroup's piece of a row

struct Sums {
  double w, p;  // of the weights, and of the target's probabilities
};

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

__device__ __forceinline__ double counted(double w) { return w > 0.0 && w < __builtin_inf() ? w : 0.0; }

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
  // those of the tokens from i on (p's own where `plain`), 0 past the vocabulary
  __device__ __forceinline__ void load(int64_t i, double (&w)[Vec<T>::n], double (&pp)[Vec<T>::n]) const {
    constexpr int n = Vec<T>::n;
    typedef typename Vec<T>::type V;
    float x[n], y[n];
    if (i + n <= vocab) {
      const V u = *reinterpret_cast<const V*>(p + i);
#pragma unroll
      for (int e = 0; e < n; ++e) x[e] = to_f32((T)u[e]);
      if (q) {
        const V v = *reinterpret_cast<const V*>(q + i);
#pragma unroll
        for (int e = 0; e < n; ++e) y[e] = to_f32((T)v[e]);
      }
    } else {
#pragma unroll
      for (int e = 0; e < n; ++e) {
        x[e] = i + e < vocab ? to_f32(p[i + e]) : 0.0f;
        y[e] = q && i + e < vocab ? to_f32(q[i + e]) : 0.0f;
      }
    }
#pragma unroll
    for (int e = 0; e < n; ++e) {
      pp[e] = counted((double)x[e]);
      w[e] = q ? counted((double)x[e] - (double)y[e]) : i + e == less ? counted((double)x[e] - 1.0) : pp[e];
    }
  }
};

__device__ __forceinline__ double sum_of_wave(double x) {
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) x += __shfl_xor(x, off, 64);
  return x;
}

template <typename T>
__global__ __launch_bounds__(kThreads) void k_verify_sums(VerifyArgs a, int pieces, int64_t n_wg, Sums* sums, int32_t* places) {
  __shared__ int64_t s_place;
  __shared__ Sums part[kThreads / 64];
  const uint32_t wg = workgroup<kThreads>();
  if (wg >= n_wg) return;
  const int s = (int)(wg / pieces), piece = (int)(wg % pieces);
  const Rows rows = rows_of(a, s);
  if (rows.n == 0) return;
  if (threadIdx.x < 64) {
    const int64_t place = place_of<T>(a, rows);
    if (threadIdx.x == 0) s_place = place;
  }
  __syncthreads();
  const int64_t place = s_place;
  const Weights<T> weights(a, rows, place);
  constexpr int n = Vec<T>::n;
  double w = 0.0, p = 0.0;
#pragma unroll 4
  for (int j = 0; j < kPiece / (kThreads * n); ++j) {
    double wv[n], pv[n];
    weights.load((int64_t)piece * kPiece + (j * kThreads + threadIdx.x) * n, wv, pv);
#pragma unroll
    for (int e = 0; e < n; ++e) {
      w += wv[e];
      p += pv[e];
    }
  }
  w = sum_of_wave(w);
  p = sum_of_wave(p);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = {w, p};
  __syncthreads();
  if (threadIdx.x == 0) {
    Sums t = part[0];
#pragma unroll
    for (int i = 1; i < kThreads / 64; ++i) {
      t.w += part[i].w;
      t.p += part[i].p;
    }
    sums[wg] = t;
    if (piece == 0) places[s] = (int32_t)place;
  }
}

// Inclusive sums over the workgroup's threads, in their order; `total` is everyone's.
__device__ __forceinline__ double scan(double x, double* wave_sums, double& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const double y = __shfl_up(x, off, 64);
    if (lane >= off) x += y;
  }
  if (lane == 63) wave_sums[wave] = x;
  __syncthreads();
  double before = 0.0;
  total = 0.0;
#pragma unroll
  for (int w = 0; w < kThreads / 64; ++w) {
    if (w < wave) before += wave_sums[w];
    total += wave_sums[w];
  }
  __syncthreads();
  return x + before;
}

template <typename T>
__global__ __launch_bounds__(kThreads) void k_verify_draw(VerifyArgs a, int pieces, const Sums* sums, const int32_t* places) {
  __shared__ double wave_sums[kThreads / 64];
  __shared__ int s_first, s_last;
  __shared__ double s_base;
  const uint32_t s = workgroup<kThreads>();
  if (s >= (uint32_t)a.n_seq) return;
  const int tid = threadIdx.x;
  const Rows rows = rows_of(a, (int)s);
  int64_t place = -1, token = -1;
  if (rows.n > 0) {
    place = places[s];
    const Weights<T> weights(a, rows, place);
    sums += (int64_t)s * pieces;
    double wt = 0.0, pt = 0.0, total;
    for (int c = tid; c < pieces; c += kThreads) {
      wt += sums[c].w;
      pt += sums[c].p;
    }
    scan(wt, wave_sums, wt);
    scan(pt, wave_sums, pt);
    const bool plain = !(wt > 0.0);  // nothing of p lies above q: p itself
    const double mark = (double)a.u[rows.begin + rows.n - 1] * (plain ? pt : wt);
    if (plain ? pt > 0.0 : true) {
      // the piece in which the running sum passes the mark, or the last one that counts
      if (tid == 0) {
        s_first = 0x7FFFFFFF;
        s_last = -1;
      }
      __syncthreads();
      double before = 0.0;
      for (int c0 = 0; c0 < pieces; c0 += kThreads) {
        const int c = c0 + tid;
        const double x = c < pieces ? (plain ? sums[c].p : sums[c].w) : 0.0;
        const double upto = before + scan(x, wave_sums, total);
        if (x > 0.0) {
          if (upto > mark) atomicMin(&s_first, c);
          atomicMax(&s_last, c);
        }
        __syncthreads();
        if (c == s_first || (s_first == 0x7FFFFFFF && c == s_last)) s_base = upto - x;
        if (s_first != 0x7FFFFFFF) break;
        before += total;
        __syncthreads();
      }
      __syncthreads();
      const int piece = s_first != 0x7FFFFFFF ? s_first : s_last;
      before = s_base;
      __syncthreads();
      if (tid == 0) {
        s_first = 0x7FFFFFFF;
        s_last = -1;
      }
      __syncthreads();
      constexpr int n = Vec<T>::n;
      for (int j = 0; j < kPiece / (kThreads * n); ++j) {
        const int at = (j * kThreads + tid) * n;
        double w[n], p[n], x = 0.0;
        weights.load((int64_t)piece * kPiece + at, w, p);
        if (plain)
#pragma unroll
          for (int e = 0; e < n; ++e) w[e] = p[e];
#pragma unroll
        for (int e = 0; e < n; ++e) x += w[e];
        double run = before + (scan(x, wave_sums, total) - x);
#pragma unroll
        for (int e = 0; e < n; ++e) {
          run += w[e];
          if (w[e] > 0.0) {
            if (run > mark) atomicMin(&s_first, at + e);
            atomicMax(&s_last, at + e);
          }
        }
        before += total;
      }
      __syncthreads();
      token = (int64_t)piece * kPiece + (s_first != 0x7FFFFFFF ? s_first : s_last);
    }
  }
  for (int64_t i = tid; i < rows.n; i += kThreads)
    a.tokens_out[rows.begin + i] = i < place ? a.tokens[rows.begin + i + 1] : i == place ? (int32_t)token : -1;
  if (tid == 0) {
    a.n_out[s] = (int32_t)(place + 1);
    if (a.keep) a.keep[s] = (int32_t)(a.kv_len[s] - rows.n + place + 1);
  }
}

int64_t pieces_of(int64_t vocab) { return (vocab + kPiece - 1) / kPiece; }

template <typename T>
hipError_t launch(const VerifyArgs& a, void* ws, hipStream_t st) {
  const int64_t pieces = pieces_of(a.vocab), n = pieces * a.n_seq;
  if (n >= (int64_t)1 << 31) return hipErrorInvalidValue;
  Sums* sums = static_cast<Sums*>(ws);
  int32_t* places = reinterpret_cast<int32_t*>(sums + n);
  hipLaunchKernelGGL((k_verify_sums<T>), grid_of<kThreads>(n), dim3(kThreads), 0, st, a, (int)pieces, n, sums, places);
  hipLaunchKernelGGL((k_verify_draw<T>), grid_of<kThreads>(a.n_seq), dim3(kThreads), 0, st, a, (int)pieces, sums, places);
  return hipGetLastError();
}

}  // namespace

size_t verify_ws_bytes(int n_seq, int64_t vocab) { return (size_t)n_seq * (pieces_of(vocab) * sizeof(Sums) + 4); }

hipError_t launch_verify(const VerifyArgs& a, void* ws, hipStream_t st) {
  if (a.dtype == AWSRC_DTYPE_F32) return launch<float>(a, ws, st);
  if (a.dtype == AWSRC_DTYPE_BF16) return launch<__bf16>(a, ws, st);
  return launch<_Float16>(a, ws, st);
}

}  // namespace awsrc
