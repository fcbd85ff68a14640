// Attention over the paged int8 cache (kv_cache.hip writes it): for query row
// i of a sequence with `len` cached tokens, of which the last `new` are the
// call's own,
//   o_i = sum_t p_it v_t,  p_i = softmax_t(scale q_i . k_t),  t <= len - new + i
// (every t < len where causal is 0), with k_t = s_K c_t and v_t = s_V c_t for
// the codes c and the scales of the token's page.  A row that sees nothing is 0.
//
// Matrix products in fp16 with fp32 sums: the codes are fp16 exactly, a query
// row is brought to magnitudes below 2 by a power of two (exact, but for
// channels 2^-14 below the row's largest), and p is at most 1 by the running
// maximum.  p is rounded to fp16's 11 bits for the second product, which takes
// the matrix cores' fp16 rate: fp16 outputs lie 2.8e-4 rms from the formula in
// 64 bits, 2.1e-4 with fp32 weights; bf16 ones 1.7e-3 either way.  The key scale
// multiplies the score.  The value scale goes into the
// exponent, p' = exp2(s + log2 s_V - max), so that p' c needs no further
// scaling and p' stays in fp16's range whatever the pages' scales are; the
// denominator sums p' / s_V in fp32.
//
// The maxima in use lag: they move only when some row of the wavefront passes its
// own by 2^8, which keeps p' far below fp16's range and spares the older sums'
// rescaling in nearly every step.
//
// Layout: the score product is taken as K Q^T and its rows are assigned to
// tokens so that a lane ends with one query's scores of 16 consecutive tokens
// (which lie in one page): the right operand of V^T P^T without any exchange
// between lanes.
//
// Two kernels: k_kv_attention_rows for up to 64 query rows of a (sequence, cached
// head), bound by the cache's bytes, and k_kv_attention_tiles for more, bound
// by the matrix cores and the exponentials.  Both may split the tokens over
// workgroups, whose sums k_kv_attention_join puts together.
#include "serve_internal.h"

namespace awsrc {

namespace {

constexpr float kLog2e = 1.44269504088896340736f;
// value scales below this are 0 (the recipe writes none between 0 and 2^-107)
constexpr float kZeroScale = 0x1p-120f;
// a page this much (log2) below the row's M adds nothing to the fp16 products
constexpr float kQuiet = 60.0f;

// Four int8 codes as fp16, exactly: c + 128 in the low byte of 1024 + x, less 1152.
__device__ __forceinline__ void codes_to_f16(uint32_t w, h2& lo, h2& hi) {
  w ^= 0x80808080u;
  const uint32_t a = __builtin_amdgcn_perm(0x64646464u, w, 0x04010400u);
  const uint32_t b = __builtin_amdgcn_perm(0x64646464u, w, 0x04030402u);
  const h2 off = {(_Float16)1152.0f, (_Float16)1152.0f};
  lo = __builtin_bit_cast(h2, a) - off;
  hi = __builtin_bit_cast(h2, b) - off;
}
__device__ __forceinline__ h8 codes_to_f16x8(uint32_t w0, uint32_t w1) {
  h2 a, b, c, d;
  codes_to_f16(w0, a, b);
  codes_to_f16(w1, c, d);
  return h8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// The running softmax of a row, over lanes that hold U runs of 16 tokens each.
template <int U>
struct Softmax {
  float m = -__builtin_inff();  // of the scores seen (times log2 e); lags behind the maximum by at most kLag
  float M = -__builtin_inff();  // of score + log2 s_V
  float off[U];                 // p' = exp2(score + off)
  float f[U];                   // p = p' f
  bool quiet[U];                // the run's page adds nothing to the output
};
constexpr float kLag = 8.0f;
// p' is kept this much (log2) above 1 at its maximum, out of fp16's subnormals
// for weights down to 2^-20 of the largest; with the lag it reaches 2^14
constexpr float kLift = 6.0f;

__device__ __forceinline__ float finite_or_zero(float m) { return m == -__builtin_inff() ? 0.0f : m; }
// The factor of (sum p' c) / (sum p) in the output.  Where every seen page's value scale is 0, M stays -inf and the
// sum p' c is 0: so is the factor, which the scores alone could take to infinity (m below -134).
__device__ __forceinline__ float output_factor(float m, float M) {
  return M == -__builtin_inff() ? 0.0f : __builtin_amdgcn_exp2f(M - kLift - finite_or_zero(m));
}

// Largest value over a row's lanes: those 16 and 32 apart (four lanes a row) or 32 apart (two).
template <int LANES>
__device__ __forceinline__ float row_max(float x) {
  if constexpr (LANES == 4) x = fmaxf(x, __shfl_xor(x, 16, 64));
  return fmaxf(x, __shfl_xor(x, 32, 64));
}

// One step: run[u] is the largest seen score of run u, of a page of value scale
// sv[u].  Where the maxima moved, returns true with the factors of the older sums.
template <int LANES, int U>
__device__ __forceinline__ bool softmax_step(Softmax<U>& s, const float (&run)[U], const float (&sv)[U], const bool (&seen)[U],
                                             float& alpha_l, float& alpha_o) {
  float lsv[U], top = -__builtin_inff(), Top = top;
  bool zero[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    zero[u] = sv[u] < kZeroScale;
    lsv[u] = __builtin_amdgcn_logf(sv[u]);  // log2
    top = fmaxf(top, run[u]);
    Top = fmaxf(Top, seen[u] && !zero[u] ? run[u] + lsv[u] : -__builtin_inff());
  }
  top = row_max<LANES>(top);
  Top = row_max<LANES>(Top);
  const bool moved = __any(top > s.m + kLag || Top > s.M + kLag);
  if (moved) {
    const float mn = fmaxf(s.m, top), Mn = fmaxf(s.M, Top);
    alpha_l = __builtin_amdgcn_exp2f(s.m - finite_or_zero(mn));
    alpha_o = __builtin_amdgcn_exp2f(s.M - finite_or_zero(Mn));
    s.m = mn;
    s.M = Mn;
  }
  const float mu = finite_or_zero(s.m), Mu = finite_or_zero(s.M) - kLift;
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const float gap = Mu - mu - lsv[u];
    s.quiet[u] = zero[u] || gap > kQuiet;
    s.off[u] = !seen[u] ? 0.0f : s.quiet[u] ? -mu : lsv[u] - Mu;
    s.f[u] = !seen[u] || s.quiet[u] ? 1.0f : __builtin_amdgcn_exp2f(gap);
  }
  return moved;
}

// Where a workgroup's query rows (row = token * group + head of the group) lie
// and how many tokens they see.
struct Rows {
  int64_t r0;     // packed row of the sequence's first token
  int n_new, G, head;
  int len, most;  // cached tokens; tokens that the table and the caller's bound reach
  int causal;
  __device__ __forceinline__ bool set(const AttentionArgs& a, int s, int h) {
    const int64_t first = a.cu[s], last = a.cu[s + 1];
    if (first < 0 || last > a.n_rows || last <= first) return false;
    r0 = first;
    n_new = (int)(last - first);
    G = a.q_heads / a.c.kv_heads;
    head = h;
    len = a.kv_len[s];
    int64_t m = a.table_ld * a.c.page_tokens;
    if (m > a.max_kv) m = a.max_kv;
    most = m < len ? (int)m : len;
    causal = a.causal;
    return true;
  }
  __device__ __forceinline__ int total() const { return n_new * G; }
  // tokens below this are seen by row R
  __device__ __forceinline__ int limit(int R) const {
    const int lim = causal ? len - n_new + R / G + 1 : len;
    return lim < most ? lim : most;
  }
  // offset of row R in a [rows][heads][D] tensor with rows ld apart
  __device__ __forceinline__ int64_t at(int R, int64_t ld, int D) const {
    const int t = R / G;
    return (r0 + t) * ld + (int64_t)(head * G + R - t * G) * D;
  }
};

constexpr int kRowTile = 16, kTileRows = 128;  // of the two kernels
constexpr int kMaxSplit = 2048, kFewSplit = 8;
struct Plan {
  int tile;                     // query rows of a workgroup
  int waves;                    // of a workgroup
  int tiles_q, n_split, chunk;  // chunk: tokens of a split
};
template <int BR>
__device__ __forceinline__ float* part_of(float* parts, int64_t index, int D) {
  return parts + index * (BR * (D + 3));  // O [BR][D], then m, M and L [BR]
}

// A query row's N values of a lane, ch(i) the channel of the i-th (8 adjacent ones at a time).
template <int N, typename T>
struct Query {
  struct alignas(16) Piece { T x[8]; };
  Piece p[N / 8];
  template <typename CH>
  __device__ __forceinline__ void fetch(const T* q, const CH& ch) {
#pragma unroll
    for (int i = 0; i < N / 8; ++i) p[i] = *reinterpret_cast<const Piece*>(q + ch(8 * i));
  }
  // As fp16 fragments below 2 in magnitude, by a power of two, times the sign of
  // the scale (0 for a row that is not live); returns the score's factor.
  template <int LANES>
  __device__ __forceinline__ float fragments(bool live, float scale, h8 (&out)[N / 8]) const {
    float qm = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) qm = amax_keep(qm, live ? to_f32(p[i >> 3].x[i & 7]) : 0.0f);
    if constexpr (LANES == 4) qm = amax_keep(qm, __shfl_xor(qm, 16, 64));
    qm = amax_keep(qm, __shfl_xor(qm, 32, 64));
    int e2 = 0;
    if (qm > 0.0f && qm < __builtin_inff()) e2 = ilogbf(qm);
    const float sign = scale < 0.0f ? -1.0f : 1.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) out[i >> 3][i & 7] = (_Float16)ldexpf(live ? to_f32(p[i >> 3].x[i & 7]) * sign : 0.0f, -e2);
    return ldexpf(fabsf(scale) * kLog2e, e2);
  }
};

// Few rows.  One workgroup: 16 query rows of one (sequence, cached head) and one
// chunk of its tokens, in tiles of 64 tokens over W wavefronts that meet in LDS at
// the end.  Keys and values go from memory to the matrix cores in 16-byte runs of
// codes per lane, without LDS: a tile's values and the next tile's keys are in
// flight while the scores and the softmax are computed.  Bound by the cache's bytes: a ragged batch of 64 sequences of
// a 32B layer (684 MB) 126 us, 5.4 TB/s; short calls by the latency of a tile's loads.
//
// Lane l holds query l % 16.  Row 4 g + i of score tile j is token 16 g + 4 j + i.
// Q and K agree on an order of the channels in which each lane reads 16
// consecutive bytes of a key: channels 64 c + 16 g + 8 h + 0..7 are step (c, h).
template <typename T, int D, int W>
__global__ __launch_bounds__(64 * W, W == 8 ? 2 : D == 256 ? 1 : 3) void k_kv_attention_rows(AttentionArgs a, Plan plan, float* parts) {
  constexpr int NC = D / 64;  // 64-channel steps of the scores
  constexpr int ND = D / 16;  // 16-channel tiles of the output
  constexpr int kTurn = 64 * W;  // tokens of a round
  __shared__ float sh_m[W][16], sh_M[W][16], sh_l[W][16];
  __shared__ float sh_o[W][16][D + 4];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = lane & 15, g = lane >> 4;
  uint32_t b = workgroup<64 * W>();
  const int qt = b % (uint32_t)plan.tiles_q;
  b /= (uint32_t)plan.tiles_q;
  const int head = b % (uint32_t)a.c.kv_heads;
  b /= (uint32_t)a.c.kv_heads;
  const int split = b % (uint32_t)plan.n_split, s = b / (uint32_t)plan.n_split;
  if (s >= a.n_seq) return;
  Rows rows;
  if (!rows.set(a, s, head)) return;
  const int R0 = qt * 16, n_rows = rows.total() - R0;
  if (n_rows <= 0) return;
  const int full = rows.limit(R0 + (n_rows < 16 ? n_rows : 16) - 1);  // tokens that any row sees
  const int start = split * plan.chunk;
  if (split && start >= full) return;
  const int end = full < start + plan.chunk ? full : start + plan.chunk;
  const bool live = r < n_rows;
  int lim = live ? rows.limit(R0 + r) : 0;
  if (lim > end) lim = end;

  Query<16 * NC, T> query;
  query.fetch(static_cast<const T*>(a.q) + rows.at(live ? R0 + r : R0, a.ldq, D),
              [&](int i) { return 64 * (i >> 4) + 16 * g + (i & 8); });
  h8 qa[2 * NC];
  const float qscale = query.template fragments<4>(live, a.scale, qa);
  Softmax<1> sm;
  float L = 0.0f;
  fl4 o[ND];
#pragma unroll
  for (int d = 0; d < ND; ++d) o[d] = fl4{0, 0, 0, 0};

  const int32_t* table = a.table + (int64_t)s * a.table_ld;
  const int shift = __builtin_ctz(a.c.page_tokens), P = a.c.page_tokens;
  const int64_t stride = (int64_t)P * D;
  // the tokens whose page a lane needs: of its value run and scores, and of its key rows; past the end the
  // tile's first token stands in (the scores are masked)
  const auto token = [&](int t0, int run) { return t0 + 16 * run < end ? t0 + 16 * run : t0; };
  u32x4_t kw[4][NC];
  float sk = 0.0f, sv = 0.0f, sk_next, sv_next;
  int64_t bv = 0, bv_next;
  bool ok = false, ok_next;
  int32_t pk = 0, pv = 0;  // pages of the tile whose keys are loaded next
  const auto pages = [&](int t0) {
    pv = table[token(t0, g) >> shift];
    pk = table[token(t0, r >> 2) >> shift];
  };
  const auto load_keys = [&](int t0) {
    ok_next = pv >= 0 && pv < a.c.n_pages;
    bv_next = (int64_t)(ok_next ? pv : 0) * a.c.kv_heads + head;
    const int64_t bk = (int64_t)(pk >= 0 && pk < a.c.n_pages ? pk : 0) * a.c.kv_heads + head;
    sk_next = a.c.k_scale[bv_next];
    sv_next = a.c.v_scale[bv_next];
    const int8_t* kb = a.c.k + bk * stride + ((token(t0, r >> 2) & (P - 1)) + (r & 3)) * D + 16 * g;
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int c = 0; c < NC; ++c) kw[j][c] = *reinterpret_cast<const u32x4_t*>(kb + 4 * j * D + 64 * c);
  };
  int t0 = start + wave * 64;
  if (t0 < end) {
    pages(t0);
    load_keys(t0);
    if (t0 + kTurn < end) pages(t0 + kTurn);
  }
  for (; t0 < end; t0 += kTurn) {
    sk = sk_next * qscale;
    sv = sv_next;
    bv = bv_next;
    ok = ok_next;
    const int8_t* vb = a.c.v + bv * stride + (int64_t)r * P + (token(t0, g) & (P - 1));
    u32x4_t vw[ND];
#pragma unroll
    for (int d = 0; d < ND; ++d) vw[d] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(vb + 16 * d * P));
    fl4 sc[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      sc[j] = fl4{0, 0, 0, 0};
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        const u32x4_t w = kw[j][c];
        sc[j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(codes_to_f16x8(w[0], w[1]), qa[2 * c], sc[j], 0, 0, 0);
        sc[j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(codes_to_f16x8(w[2], w[3]), qa[2 * c + 1], sc[j], 0, 0, 0);
      }
    }
    if (t0 + kTurn < end) {
      load_keys(t0 + kTurn);
      if (t0 + 2 * kTurn < end) pages(t0 + 2 * kTurn);
    }
    // how many of the lane's 16 tokens are seen
    const int left = ok ? lim - (t0 + 16 * g) : 0;
    // unseen scores become -inf: no product of one with 0 (2^-120 does as well) or NaN
    sk = left <= 0 ? 1.0f : sk == 0.0f ? 0x1p-120f : sk;
    if (!__all(left >= 16 || !live)) {
      asm volatile("");  // keeps this a branch: nearly every tile is seen whole
#pragma unroll
      for (int e = 0; e < 16; ++e) sc[e >> 2][e & 3] = e < left ? sc[e >> 2][e & 3] : -__builtin_inff();
    }
    float x = sc[0][0];
#pragma unroll
    for (int e = 1; e < 16; ++e) x = fmaxf(x, sc[e >> 2][e & 3]);
    float alpha_l, alpha_o;
    if (softmax_step<4, 1>(sm, {x * sk}, {sv}, {left > 0}, alpha_l, alpha_o)) {
      L *= alpha_l;
#pragma unroll
      for (int d = 0; d < ND; ++d) o[d] *= alpha_o;
    }
    float p[16], l = 0.0f;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      p[e] = __builtin_amdgcn_exp2f(sc[e >> 2][e & 3] * sk + sm.off[0]);
      l += p[e];
    }
    L += l * sm.f[0];
    h8 ph[2];
#pragma unroll
    for (int e = 0; e < 16; ++e) ph[e >> 3][e & 7] = (_Float16)p[e];
    if (__any(sm.quiet[0])) {
      if (sm.quiet[0]) ph[0] = ph[1] = h8{0, 0, 0, 0, 0, 0, 0, 0};
    }
#pragma unroll
    for (int d = 0; d < ND; ++d) {
      const u32x4_t x = vw[d];
      o[d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(codes_to_f16x8(x[0], x[1]), ph[0], o[d], 0, 0, 0);
      o[d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(codes_to_f16x8(x[2], x[3]), ph[1], o[d], 0, 0, 0);
    }
  }
  L += __shfl_xor(L, 16, 64);
  L += __shfl_xor(L, 32, 64);
  if (g == 0) {
    sh_m[wave][r] = sm.m;
    sh_M[wave][r] = sm.M;
    sh_l[wave][r] = L;
  }
#pragma unroll
  for (int d = 0; d < ND; ++d) *reinterpret_cast<fl4*>(&sh_o[wave][r][16 * d + 4 * g]) = o[d];
  __syncthreads();
  const bool whole = full <= plan.chunk;  // this workgroup saw every token
  float* part = part_of<16>(parts, ((int64_t)(s * a.c.kv_heads + head) * plan.tiles_q + qt) * plan.n_split + split, D);
  for (int i = threadIdx.x; i < 16 * D / 4; i += 64 * W) {
    const int row = i / (D / 4), d = (i - row * (D / 4)) * 4;
    if (row >= n_rows) break;
    float m = -__builtin_inff(), M = m;
#pragma unroll
    for (int w = 0; w < W; ++w) {
      m = fmaxf(m, sh_m[w][row]);
      M = fmaxf(M, sh_M[w][row]);
    }
    const float mu = finite_or_zero(m), Mu = finite_or_zero(M);
    float l = 0.0f;
    fl4 y = {0, 0, 0, 0};
#pragma unroll
    for (int w = 0; w < W; ++w) {
      l += __builtin_amdgcn_exp2f(sh_m[w][row] - mu) * sh_l[w][row];
      y += __builtin_amdgcn_exp2f(sh_M[w][row] - Mu) * *reinterpret_cast<const fl4*>(&sh_o[w][row][d]);
    }
    if (whole) {
      const float f = output_factor(m, M);
      struct alignas(8) Four { T v[4]; } out;
#pragma unroll
      for (int e = 0; e < 4; ++e) out.v[e] = (T)(l == 0.0f ? 0.0f : y[e] / l * f);
      *reinterpret_cast<Four*>(static_cast<T*>(a.out) + rows.at(R0 + row, a.ldo, D) + d) = out;
    } else {
      *reinterpret_cast<fl4*>(part + row * D + d) = y;
      if (d == 0) {
        part[16 * D + row] = m;
        part[16 * D + 16 + row] = M;
        part[16 * D + 32 + row] = l;
      }
    }
  }
}

template <typename T>
__device__ __forceinline__ void store_row4(T* out, fl4 y, float l, float f) {
  struct alignas(8) Four { T v[4]; } w;
#pragma unroll
  for (int e = 0; e < 4; ++e) w.v[e] = (T)(l == 0.0f ? 0.0f : y[e] / l * f);
  *reinterpret_cast<Four*>(out) = w;
}

// Many rows.  One workgroup: 32 W query rows of one (sequence, cached head), 32 a
// wavefront, over tiles of 64 tokens whose codes become fp16 once, on their way
// into LDS (two stages), and then serve all W wavefronts through 32 x 32 x 16
// products.  The next tile's codes are on their way from memory while the
// current one is computed.  Bound by vector and matrix instructions one after the
// other (8192 tokens of a 3B layer: 320 us, 860 TFLOP/s, 315 to 330 by machine; of the CUs' busy cycles 58% issue
// vector instructions and 39% run matrix ones).  Neither wavefront priorities, nor half
// of the wavefronts a phase behind the others, nor the next tile's scores during this one's exponentials (too many
// registers) overlapped them: four SIMDs at their products take LDS's whole rate, 1 KB in 32 cycles each.
//
// Lane l (half h = l / 32) holds query l % 32.  Row 8 b + 4 h + i of a 32-token score
// tile is token 16 h + 4 b + i.  Keys lie in LDS as [row][channel], values as
// [channel][token], in pieces of 16 bytes at place p ^ key(row), so that the 16
// lanes that LDS serves at once, reading one piece of 16 rows, meet all its banks.
__device__ __forceinline__ int value_key(int d) { return (d >> 1) & 7; }
template <int D>
struct TileLds {
  static __device__ __forceinline__ int key(int row) { return D == 64 ? (row >> 1) & 7 : row & 15; }
  static constexpr int kKeys = 64 * D * 2, kValues = D * 64 * 2;
  static constexpr int kStage = kKeys + kValues;
  // by 16-token run: of the two stages the scales and the page (negative: none), of the two tiles to come where
  // their codes start and the page
  float run_k[2][4], run_v[2][4];
  int run_page[2][4], next_page[2][4];
  int64_t next_k[2][4], next_v[2][4];
};

// The order of a block of N matrix products, consecutive ones on different sums: every operand is read from LDS four
// products ahead.  8192 tokens of a 3B layer: 320 us, 325 in the compiler's own order.
template <int N>
__device__ __forceinline__ void reads_ahead() {
  constexpr int kProduct = 0x8, kRead = 0x100;
  __builtin_amdgcn_sched_group_barrier(kRead, 6, 0);  // (two may be others of the block)
#pragma unroll
  for (int i = 0; i < N - 4; ++i) {
    __builtin_amdgcn_sched_group_barrier(kProduct, 1, 0);
    __builtin_amdgcn_sched_group_barrier(kRead, 1, 0);
  }
  __builtin_amdgcn_sched_group_barrier(kProduct, 4, 0);
}

template <typename T, int D, int W>
__global__ __launch_bounds__(64 * W, D == 256 ? 1 : 2) void k_kv_attention_tiles(AttentionArgs a, Plan plan, float* parts) {
  constexpr int BR = 32 * W;
  constexpr int kThreads = 64 * W;
  constexpr int NS = D / 16;   // 16-channel steps of the scores
  constexpr int ND = D / 32;   // 32-channel tiles of the output
  constexpr int NL = D * 4 / kThreads;  // 16-byte runs of codes a thread moves per tile, of keys and of values
  static_assert(NL >= 1 && NL * kThreads == D * 4, "runs of a tile");
  using S = TileLds<D>;
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  S& sh = *reinterpret_cast<S*>(lds + 2 * S::kStage);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r = lane & 31, h = lane >> 5;
  uint32_t b = workgroup<64 * W>();
  const int head = b % (uint32_t)a.c.kv_heads;
  b /= (uint32_t)a.c.kv_heads;
  // the last rows see the most tokens: they start first
  const int qt = plan.tiles_q - 1 - (int)(b % (uint32_t)plan.tiles_q);
  b /= (uint32_t)plan.tiles_q;
  // every sequence's first part before any second: the short last parts start late (pieces of 601 tokens in seven
  // sequences of up to 6007, heads of 64: 123 us sequence by sequence, 120; of a 32B layer 513 and 508)
  const int s = b % (uint32_t)a.n_seq, split = b / (uint32_t)a.n_seq;
  if (split >= plan.n_split) return;
  Rows rows;
  if (!rows.set(a, s, head)) return;
  const int R0 = qt * BR, n_rows = rows.total() - R0;
  if (n_rows <= 0) return;
  const int full = rows.limit(R0 + (n_rows < BR ? n_rows : BR) - 1);
  const int start = split * plan.chunk;
  if (split && start >= full) return;
  const int end = full < start + plan.chunk ? full : start + plan.chunk;
  const int R = R0 + wave * 32 + r;
  const bool live = wave * 32 + r < n_rows;
  int lim = live ? rows.limit(R) : 0;
  if (lim > end) lim = end;
  // tokens that every row of the wavefront sees: tiles below need no masks
  int all = rows.limit(R0 + wave * 32 < rows.total() ? R0 + wave * 32 : rows.total() - 1);
  if (all > end) all = end;
  // tokens that any row of the wavefront sees
  const int top_row = R0 + wave * 32 + 31 < rows.total() ? R0 + wave * 32 + 31 : rows.total() - 1;
  int any = wave * 32 < n_rows ? rows.limit(top_row) : 0;
  if (any > end) any = end;

  Query<8 * NS, T> query;
  query.fetch(static_cast<const T*>(a.q) + rows.at(live ? R : R0, a.ldq, D), [&](int i) { return 2 * i + 8 * h; });
  h8 qa[NS];
  const float qscale = query.template fragments<2>(live, a.scale, qa);

  const int32_t* table = a.table + (int64_t)s * a.table_ld;
  const int P = a.c.page_tokens, shift = __builtin_ctz(P);
  const int64_t stride = (int64_t)P * D;
  // this thread's runs: of keys, token (tid + kThreads i) / (D / 16) from channel 16 (tid % (D / 16)); of values,
  // channel (tid + kThreads i) / 4, tokens from 16 (tid % 4)
  constexpr int KR = D / 16;
  // where the codes of a tile's runs start, by its first four threads, into place `slot` of the ring; tokens past the
  // end take the tile's first page (masked)
  const auto find = [&](int t0, int slot) {
    const int t = t0 + 16 * tid < end ? t0 + 16 * tid : t0;
    int page = table[t >> shift];
    if (page < 0 || page >= a.c.n_pages) page = -1;
    const int64_t block = ((int64_t)(page < 0 ? 0 : page) * a.c.kv_heads + head) * stride;
    sh.next_page[slot][tid] = page;
    sh.next_k[slot][tid] = block + (t & (P - 1)) * D;
    sh.next_v[slot][tid] = block + (t & (P - 1));
  };
  u32x4_t kw[NL], vw[NL];
  float gk = 0.0f, gv = 0.0f;
  int gp = -1;
  const int8_t* k_mine = a.c.k + ((tid / KR) & 15) * D + 16 * (tid % KR);
  const int8_t* v_mine = a.c.v + (int64_t)(tid >> 2) * P;
  const auto load = [&](int slot) {
#pragma unroll
    for (int i = 0; i < NL; ++i)  // kThreads / KR tokens on: a whole number of runs
      kw[i] = *reinterpret_cast<const u32x4_t*>(k_mine + sh.next_k[slot][(tid + kThreads * i) / KR >> 4]);
    const int8_t* vb = v_mine + sh.next_v[slot][tid & 3];
#pragma unroll
    for (int i = 0; i < NL; ++i) vw[i] = *reinterpret_cast<const u32x4_t*>(vb + (int64_t)(kThreads / 4 * i) * P);
    if (tid < 4) {
      gp = sh.next_page[slot][tid];
      const int64_t block = (int64_t)(gp < 0 ? 0 : gp) * a.c.kv_heads + head;
      gk = a.c.k_scale[block];
      gv = a.c.v_scale[block];
    }
  };
  const auto store = [&](int stage) {
    char* base = lds + stage * S::kStage;
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const int x = tid + kThreads * i, t = x / KR, c = x % KR;
      // token 32 u + 16 h + 4 b + e is row 32 u + 8 b + 4 h + e
      const int row = (t & 32) | ((t >> 2) & 3) << 3 | ((t >> 4) & 1) << 2 | (t & 3);
      char* o = base + row * 2 * D;
      *reinterpret_cast<h8*>(o + ((2 * c) ^ S::key(row)) * 16) = codes_to_f16x8(kw[i][0], kw[i][1]);
      *reinterpret_cast<h8*>(o + ((2 * c + 1) ^ S::key(row)) * 16) = codes_to_f16x8(kw[i][2], kw[i][3]);
    }
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const int x = tid + kThreads * i, d = x >> 2, g = x & 3;
      char* o = base + S::kKeys + d * 128;
      *reinterpret_cast<h8*>(o + ((2 * g) ^ value_key(d)) * 16) = codes_to_f16x8(vw[i][0], vw[i][1]);
      *reinterpret_cast<h8*>(o + ((2 * g + 1) ^ value_key(d)) * 16) = codes_to_f16x8(vw[i][2], vw[i][3]);
    }
    if (tid < 4) {
      sh.run_k[stage][tid] = gk;
      sh.run_v[stage][tid] = gv;
      sh.run_page[stage][tid] = gp;
    }
  };

  Softmax<2> sm;
  float L = 0.0f;
  fl16 o[ND];
#pragma unroll
  for (int d = 0; d < ND; ++d)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[d][e] = 0.0f;

  if (start < end) {  // (uniform)
    if (tid < 4) {
      find(start, 0);
      if (start + 64 < end) find(start + 64, 1);
    }
    __syncthreads();
    load(0);
    store(0);
    __syncthreads();
  }
  int stage = 0;
  for (int t0 = start; t0 < end; t0 += 64, stage ^= 1) {
    const bool more = t0 + 64 < end;
    if (more) {
      load(stage ^ 1);
      if (tid < 4 && t0 + 128 < end) find(t0 + 128, stage);  // (read a round ago)
    }
    if (t0 < any) {
      const char* base = lds + stage * S::kStage;
      fl16 sc[2];
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int e = 0; e < 16; ++e) sc[u][e] = 0.0f;
#pragma unroll
      for (int k = 0; k < NS; ++k)
#pragma unroll
        for (int u = 0; u < 2; ++u)
          sc[u] = __builtin_amdgcn_mfma_f32_32x32x16_f16(
              *reinterpret_cast<const h8*>(base + (32 * u + r) * 2 * D + ((2 * k + h) ^ S::key(r)) * 16), qa[k], sc[u], 0, 0, 0);
      reads_ahead<2 * NS>();
      float sk[2], sv[2], run[2];
      bool seen[2];
      int left[2];
      bool whole = t0 + 64 <= all;
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int g = 2 * u + h;
        const bool ok = sh.run_page[stage][g] >= 0;
        whole = whole && ok;
        left[u] = ok ? lim - (t0 + 32 * u + 16 * h) : 0;
        seen[u] = left[u] > 0;
        // unseen scores become -inf: no product of one with 0 (2^-120 does as well) or NaN
        sk[u] = sh.run_k[stage][g] * qscale;
        sk[u] = !seen[u] ? 1.0f : sk[u] == 0.0f ? 0x1p-120f : sk[u];
        sv[u] = sh.run_v[stage][g];
      }
      if (!__all(whole)) {
        asm volatile("");  // keeps this a branch: nearly every tile is seen whole
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int e = 0; e < 16; ++e) sc[u][e] = e < left[u] ? sc[u][e] : -__builtin_inff();
      }
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        float x = sc[u][0];
#pragma unroll
        for (int e = 1; e < 16; ++e) x = fmaxf(x, sc[u][e]);
        run[u] = x * sk[u];
      }
      float alpha_l, alpha_o;
      if (softmax_step<2, 2>(sm, run, sv, seen, alpha_l, alpha_o)) {
        L *= alpha_l;
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
          for (int e = 0; e < 16; ++e) o[d][e] *= alpha_o;
      }
      h8 ph[2][2];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        // summed in fp32 before the rounding: p' of a page much quieter than the row's loudest may be 0 in fp16
        // and still weigh in the denominator
        float l = 0.0f;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const float p = __builtin_amdgcn_exp2f(sc[u][e] * sk[u] + sm.off[u]);
          l += p;
          ph[u][e >> 3][e & 7] = (_Float16)p;
        }
        L += l * sm.f[u];
      }
      if (__any(sm.quiet[0] || sm.quiet[1])) {
#pragma unroll
        for (int u = 0; u < 2; ++u)
          if (sm.quiet[u]) ph[u][0] = ph[u][1] = h8{0, 0, 0, 0, 0, 0, 0, 0};
      }
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int d = 0; d < ND; ++d)
          o[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(
              *reinterpret_cast<const h8*>(base + S::kKeys + (32 * d + r) * 128 +
                                           ((4 * (j >> 1) + 2 * h + (j & 1)) ^ value_key(r)) * 16),
              ph[j >> 1][j & 1], o[d], 0, 0, 0);
      reads_ahead<4 * ND>();
    }
    if (more) store(stage ^ 1);
    __syncthreads();
  }
  L += __shfl_xor(L, 32, 64);
  if (!live) return;
  // lane: channels 32 d + 8 b + 4 h + e of its query
  if (full <= plan.chunk) {
    const float f = output_factor(sm.m, sm.M);
    T* out = static_cast<T*>(a.out) + rows.at(R, a.ldo, D) + 4 * h;
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
      for (int e = 0; e < 16; e += 4)
        store_row4(out + 32 * d + 2 * e, fl4{o[d][e], o[d][e + 1], o[d][e + 2], o[d][e + 3]}, L, f);
  } else {
    float* part = part_of<BR>(parts, ((int64_t)(s * a.c.kv_heads + head) * plan.tiles_q + qt) * plan.n_split + split, D);
    const int row = wave * 32 + r;
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
      for (int e = 0; e < 16; e += 4)
        *reinterpret_cast<fl4*>(part + row * D + 32 * d + 2 * e + 4 * h) = fl4{o[d][e], o[d][e + 1], o[d][e + 2], o[d][e + 3]};
    if (h == 0) {
      part[BR * D + row] = sm.m;
      part[BR * D + BR + row] = sm.M;
      part[BR * D + 2 * BR + row] = L;
    }
  }
}

// The sums of a row's splits together, for up to kFewSplit of them: D / 4 lanes a
// row, every lane with all statistics, so that all loads go out at once and no
// lane waits for another.  Bound by the sums' bytes (ragged pieces of prompts: 12 us, near 5 TB/s).
template <int BR, typename T, int D>
__global__ __launch_bounds__(256) void k_kv_attention_join_few(AttentionArgs a, Plan plan, const float* parts, int n_items,
                                                               int per_head) {
  constexpr int LD = D / 4;
  const int item = (int)blockIdx.x * (256 / LD) + threadIdx.x / LD, d = (threadIdx.x % LD) * 4;
  if (item >= n_items) return;
  const int sh = item / per_head, s = sh / a.c.kv_heads, R = item - sh * per_head;
  Rows rows;
  if (!rows.set(a, s, sh - s * a.c.kv_heads) || R >= rows.total()) return;
  const int qt = R / BR, row = R - qt * BR;
  const int last = qt * BR + BR - 1 < rows.total() ? qt * BR + BR - 1 : rows.total() - 1;
  if (rows.limit(last) <= plan.chunk) return;  // written whole
  const int lim = rows.limit(R), n = lim <= 0 ? 0 : (lim + plan.chunk - 1) / plan.chunk;
  const float* base = part_of<BR>(const_cast<float*>(parts), ((int64_t)sh * plan.tiles_q + qt) * plan.n_split, D);
  float m[kFewSplit], M[kFewSplit], l[kFewSplit];
  fl4 y[kFewSplit];
#pragma unroll
  for (int i = 0; i < kFewSplit; ++i) {
    const float* p = base + (int64_t)(i < n ? i : 0) * (BR * (D + 3));  // (split 0 is there whenever a row was split)
    m[i] = p[BR * D + row];
    M[i] = p[BR * D + BR + row];
    l[i] = p[BR * D + 2 * BR + row];
    y[i] = *reinterpret_cast<const fl4*>(p + row * D + d);
  }
  float mx = -__builtin_inff(), Mx = mx;
#pragma unroll
  for (int i = 0; i < kFewSplit; ++i) {
    mx = fmaxf(mx, m[i]);
    Mx = fmaxf(Mx, M[i]);
  }
  const float mu = finite_or_zero(mx), Mu = finite_or_zero(Mx);
  float sum = 0.0f;
  fl4 o = {0, 0, 0, 0};
#pragma unroll
  for (int i = 0; i < kFewSplit; ++i)
    if (i < n) {
      sum += l[i] * __builtin_amdgcn_exp2f(m[i] - mu);
      o += y[i] * __builtin_amdgcn_exp2f(M[i] - Mu);
    }
  store_row4(static_cast<T*>(a.out) + rows.at(R, a.ldo, D) + d, o, sum, output_factor(mx, Mx));
}

// The same for more splits: a workgroup per row weighs them by their maxima
// first, so that the sums' loads do not wait for one another.  128 splits of 32 rows: 5.9 us, latency.
template <int BR, typename T, int D>
__global__ __launch_bounds__(256) void k_kv_attention_join(AttentionArgs a, Plan plan, const float* parts, int per_head) {
  constexpr int LD = D / 4;    // lanes across a row
  constexpr int NP = 256 / LD; // splits summed at once
  __shared__ float sh_w[kMaxSplit];
  __shared__ float sh_s[4][3];
  __shared__ fl4 sh_o[NP][LD];
  const int t = threadIdx.x, wave = t >> 6;
  const int sh = (int)blockIdx.x / per_head, s = sh / a.c.kv_heads, R = (int)blockIdx.x - sh * per_head;
  Rows rows;
  if (!rows.set(a, s, sh - s * a.c.kv_heads) || R >= rows.total()) return;
  const int qt = R / BR, row = R - qt * BR;
  const int last = qt * BR + BR - 1 < rows.total() ? qt * BR + BR - 1 : rows.total() - 1;
  if (rows.limit(last) <= plan.chunk) return;  // written whole
  const int lim = rows.limit(R), n = lim <= 0 ? 0 : (lim + plan.chunk - 1) / plan.chunk;
  const float* base = part_of<BR>(const_cast<float*>(parts), ((int64_t)sh * plan.tiles_q + qt) * plan.n_split, D);
  const int64_t step = BR * (D + 3);
  float m = -__builtin_inff(), M = m;
  for (int i = t; i < n; i += 256) {
    const float* p = base + i * step + BR * D + row;
    m = fmaxf(m, p[0]);
    M = fmaxf(M, p[BR]);
  }
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) {
    m = fmaxf(m, __shfl_xor(m, off, 64));
    M = fmaxf(M, __shfl_xor(M, off, 64));
  }
  if ((t & 63) == 0) {
    sh_s[wave][0] = m;
    sh_s[wave][1] = M;
  }
  __syncthreads();
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    m = fmaxf(m, sh_s[w][0]);
    M = fmaxf(M, sh_s[w][1]);
  }
  const float mu = finite_or_zero(m), Mu = finite_or_zero(M);
  float l = 0.0f;
  for (int i = t; i < n; i += 256) {
    const float* p = base + i * step + BR * D + row;
    l += p[2 * BR] * __builtin_amdgcn_exp2f(p[0] - mu);
    sh_w[i] = __builtin_amdgcn_exp2f(p[BR] - Mu);
  }
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) l += __shfl_xor(l, off, 64);
  if ((t & 63) == 0) sh_s[wave][2] = l;
  __syncthreads();
  const int g = t / LD, d = t % LD;
  fl4 y = {0, 0, 0, 0};
#pragma unroll 8
  for (int i = g; i < n; i += NP) y += sh_w[i] * *reinterpret_cast<const fl4*>(base + i * step + row * D + 4 * d);
  sh_o[g][d] = y;
  __syncthreads();
  if (g) return;
#pragma unroll
  for (int i = 1; i < NP; ++i) y += sh_o[i][d];
  l = sh_s[0][2] + sh_s[1][2] + sh_s[2][2] + sh_s[3][2];
  store_row4(static_cast<T*>(a.out) + rows.at(R, a.ldo, D) + 4 * d, y, l, output_factor(m, M));
}

// Which kernel, and how the tokens are split.
Plan plan_of(const AttentionArgs& a) {
  const int64_t rows = a.max_new * (a.q_heads / a.c.kv_heads);
  Plan p;
  p.tile = rows > 64 ? kTileRows : kRowTile;
  p.tiles_q = (int)((rows + p.tile - 1) / p.tile);
  const int64_t base = (int64_t)a.n_seq * a.c.kv_heads * p.tiles_q;
  int64_t most = a.table_ld * a.c.page_tokens;
  if (most > a.max_kv) most = a.max_kv;
  // Splits, as far as they fill the machine: each costs a join.  Few rows: as many
  // workgroups as reside at once on half of the CUs' registers (D = 128: 2 x 131071 tokens of a
  // group of 8 take 29.4 us in 512 workgroups, 33.9 in 1024; the ragged batch of 64 126, 138),
  // of at least 256 tokens (2000 tokens: 10.3 us, 11.8 with 512).  Many rows: one sequence
  // 512 workgroups (512 rows after 16000 tokens: 110 us, 133 in 1024), a batch, whose lengths differ,
  // 4096 of at least 1024 tokens (pieces of 601 tokens in seven sequences of up to 6007, heads of 64:
  // 120 us, 169 in 512; of a 3B layer, where it costs, 231 and 209).
  int64_t target, least;
  if (p.tile == kRowTile) {
    target = a.c.head_dim == 64 ? 768 : a.c.head_dim == 128 ? 512 : 256;
    least = 256;
  } else {
    target = a.n_seq == 1 ? 512 : 4096;
    least = a.n_seq == 1 ? 512 : 1024;
  }
  int64_t split = p.tile == kTileRows ? target / base : (target + base - 1) / base;
  const int64_t cap = (most + least - 1) / least;
  if (split > cap) split = cap;
  // Sequences of different lengths leave CUs idle at the end: where they have to be split at all, into twice as many
  // parts, unless those get short.  Of up to 8192 tokens of a 32B layer, on the GPU in us with and without: 24 sequences
  // 54 and 63, 32 70 and 65, 40 79 and 88, 48 92 and 91, 56 114 and 126, 63 128 and 134; 64, which fill the machine
  // and stay whole, 126.
  if (p.tile == kRowTile && a.n_seq > 1 && base < target) {
    int64_t even = (2 * target + base - 1) / base;
    if (even > most / (8 * a.c.head_dim)) even = most / (8 * a.c.head_dim);
    if (split < even) split = even;
  }
  if (split > kMaxSplit) split = kMaxSplit;
  if (split < 1) split = 1;
  p.waves = 4;
  // A short history and few sequences: eight wavefronts and no split cost less than the second
  // launch does (1501 tokens: 13.3 us on the GPU and 10.4 on the host, 10.0 and 14.9 split; 2000: 16.1 and 10.0).
  if (p.tile == kRowTile && split > 1 && most <= 1536 && a.c.head_dim <= 128) {
    p.waves = 8;
    split = 1;
  }
  const int64_t chunk = ((most + split - 1) / split + 255) / 256 * 256;
  p.chunk = (int)(chunk < 256 ? 256 : chunk);
  p.n_split = (int)((most + p.chunk - 1) / p.chunk);
  if (p.n_split < 1) p.n_split = 1;
  // Rows enough for every CU twice without a split: 256 a workgroup, which halves the work of turning
  // codes into fp16 (8192 tokens of a 3B layer: 358 us with 128, 320; 1000 tokens each of four
  // sequences of a 32B layer, where whole workgroups of the shorter ones idle, 67 and 71).
  if (p.tile == kTileRows && p.n_split == 1 && a.c.head_dim == 128 && rows >= 16384) {
    const int64_t wide = (rows + 2 * kTileRows - 1) / (2 * kTileRows);
    if ((int64_t)a.n_seq * a.c.kv_heads * wide >= 512) {
      p.tile = 2 * kTileRows;
      p.waves = 8;
      p.tiles_q = (int)wide;
    }
  }
  return p;
}

template <int BR, typename T, int D>
hipError_t launch_join(const AttentionArgs& a, const Plan& p, const float* parts, hipStream_t st) {
  const int64_t per_head = a.max_new * (a.q_heads / a.c.kv_heads), items = (int64_t)a.n_seq * a.c.kv_heads * per_head;
  if (items > 0x7FFFFFFF) return hipErrorInvalidValue;
  if (p.n_split <= kFewSplit)
    hipLaunchKernelGGL((k_kv_attention_join_few<BR, T, D>), dim3((unsigned)((items * (D / 4) + 255) / 256)), dim3(256), 0, st, a, p,
                       parts, (int)items, (int)per_head);
  else
    hipLaunchKernelGGL((k_kv_attention_join<BR, T, D>), dim3((unsigned)items), dim3(256), 0, st, a, p, parts, (int)per_head);
  return hipGetLastError();
}

template <typename T, int D, int W>
hipError_t launch_tiles(const AttentionArgs& a, const Plan& p, int64_t grid, float* parts, hipStream_t st) {
  const auto k = k_kv_attention_tiles<T, D, W>;
  constexpr int bytes = 2 * TileLds<D>::kStage + sizeof(TileLds<D>);
  if (bytes > 65536) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(k), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL(k, grid_of<64 * W>(grid), dim3(64 * W), bytes, st, a, p, parts);
  return hipGetLastError();
}

template <typename T, int D>
hipError_t launch_d(const AttentionArgs& a, float* parts, hipStream_t st) {
  const Plan p = plan_of(a);
  const int64_t grid = (int64_t)a.n_seq * a.c.kv_heads * p.tiles_q * p.n_split;
  if (grid > 0x7FFFFFFF) return hipErrorInvalidValue;
  if (p.tile == kRowTile) {
    if constexpr (D <= 128) {
      if (p.waves == 8) {
        hipLaunchKernelGGL((k_kv_attention_rows<T, D, 8>), grid_of<512>(grid), dim3(512), 0, st, a, p, parts);
        return hipGetLastError();
      }
    }
    hipLaunchKernelGGL((k_kv_attention_rows<T, D, 4>), grid_of<256>(grid), dim3(256), 0, st, a, p, parts);
    if (p.n_split > 1) return launch_join<kRowTile, T, D>(a, p, parts, st);
    return hipGetLastError();
  }
  if constexpr (D == 128)
    if (p.waves == 8) return launch_tiles<T, D, 8>(a, p, grid, parts, st);
  const hipError_t e = launch_tiles<T, D, 4>(a, p, grid, parts, st);
  return e == hipSuccess && p.n_split > 1 ? launch_join<kTileRows, T, D>(a, p, parts, st) : e;
}

template <typename T>
hipError_t launch(const AttentionArgs& a, float* parts, hipStream_t st) {
  if (a.c.head_dim == 64) return launch_d<T, 64>(a, parts, st);
  if (a.c.head_dim == 128) return launch_d<T, 128>(a, parts, st);
  return launch_d<T, 256>(a, parts, st);
}

}  // namespace

size_t kv_attention_ws_bytes(const AttentionArgs& a) {
  const Plan p = plan_of(a);
  if (p.n_split == 1) return 0;
  return (size_t)a.n_seq * a.c.kv_heads * p.tiles_q * p.n_split * p.tile * (a.c.head_dim + 3) * 4;
}

hipError_t launch_kv_attention(const AttentionArgs& a, void* ws, hipStream_t st) {
  float* parts = static_cast<float*>(ws);
  return a.dtype == AWSRC_DTYPE_BF16 ? launch<__bf16>(a, parts, st) : launch<_Float16>(a, parts, st);
}

}  // namespace awsrc
