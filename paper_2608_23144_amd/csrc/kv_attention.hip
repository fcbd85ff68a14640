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
// maximum.  The key scale multiplies the score.  The value scale goes into the
// exponent, p' = exp2(s + log2 s_V - max), so that p' c needs no further
// scaling and p' stays in fp16's range whatever the pages' scales are; the
// denominator sums p' / s_V in fp32.
//
// Layout: the score product is taken as K Q^T, a lane l ending with query
// l % 16 and four tokens per 16-token tile.  Key rows are assigned to the
// tiles so that the 16 scores of a lane over four tiles are the 16
// consecutive tokens 16 (l / 16) .. + 15: the right operand of V^T P^T
// without any exchange between lanes, against V^T codes read in 16-byte runs
// of tokens.  Likewise Q and K agree on an order of the channels in which
// each lane reads 16 consecutive bytes of a key.
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

__device__ __forceinline__ float max_over_groups(float m) {
  m = fmaxf(m, __shfl_xor(m, 16, 64));
  return fmaxf(m, __shfl_xor(m, 32, 64));
}
__device__ __forceinline__ float sum_over_groups(float s) {
  s += __shfl_xor(s, 16, 64);
  return s + __shfl_xor(s, 32, 64);
}

__device__ __forceinline__ float finite_or_zero(float m) { return m == -__builtin_inff() ? 0.0f : m; }

// One step of the running softmax of a row: `run` is the largest seen score
// (times log2 e) of the lane's 16 tokens, which lie in one page of value scale
// sv; the row's other lanes hold other tokens.  Updates the row's m and M.
struct Softmax {
  float off;               // p' = exp2(s + off)
  float f;                 // p = p' f
  float alpha_l, alpha_o;  // the older sums' factors
  bool quiet;              // the page adds nothing to the output
};
__device__ __forceinline__ Softmax softmax_step(float run, float sv, bool seen, float& m, float& M) {
  const bool zero = sv < kZeroScale;
  const float lsv = __builtin_amdgcn_logf(sv);  // log2
  const float mn = fmaxf(m, max_over_groups(run));
  const float Mn = fmaxf(M, max_over_groups(seen && !zero ? run + lsv : -__builtin_inff()));
  const float mu = finite_or_zero(mn), Mu = finite_or_zero(Mn);
  const float gap = Mu - mu - lsv;
  Softmax w;
  w.quiet = zero || gap > kQuiet;
  w.off = !seen ? 0.0f : w.quiet ? -mu : lsv - Mu;
  w.f = !seen || w.quiet ? 1.0f : __builtin_amdgcn_exp2f(gap);
  w.alpha_l = __builtin_amdgcn_exp2f(m - mu);
  w.alpha_o = __builtin_amdgcn_exp2f(M - Mu);
  m = mn;
  M = Mn;
  return w;
}

// One workgroup: 16 query rows (row = token * group + head of the group) of one
// (sequence, cached head); the tokens in tiles of 64 over its 4 wavefronts,
// joined through LDS at the end.
template <typename T, int D>
__global__ __launch_bounds__(256) void k_kv_attention_rows(AttentionArgs a, int64_t tiles_q) {
  constexpr int NC = D / 64;  // 64-channel steps of the scores
  constexpr int ND = D / 16;  // 16-channel tiles of the output
  __shared__ float sh_m[4][16], sh_M[4][16], sh_l[4][16];
  __shared__ float sh_o[4][16][D + 4];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int r = lane & 15, g = lane >> 4;
  int64_t b = blockIdx.x;
  const int head = (int)(b % a.c.kv_heads);
  b /= a.c.kv_heads;
  const int64_t qt = b % tiles_q;
  const int s = (int)(b / tiles_q);
  const int G = a.q_heads / a.c.kv_heads;
  const int P = a.c.page_tokens;
  const int64_t r0 = a.cu[s], r1 = a.cu[s + 1];
  if (r0 < 0 || r1 > a.n_rows) return;
  const int64_t n_new = r1 - r0;
  if (qt * 16 >= n_new * G) return;
  const int64_t len = a.kv_len[s];
  int64_t most = a.table_ld * P;  // tokens the table and the caller's bound reach
  if (most > a.max_kv) most = a.max_kv;
  if (most > len) most = len;

  const int64_t R = qt * 16 + r;
  const bool live = R < n_new * G;
  const int64_t tok = live ? R / G : 0;
  const int qh = head * G + (int)(live ? R - tok * G : 0);
  // tokens below lim are seen
  int64_t lim = a.causal ? len - n_new + tok + 1 : len;
  if (lim > most) lim = most;
  if (!live) lim = 0;
  int64_t end = lim;  // tokens any row of the workgroup sees
#pragma unroll
  for (int off = 8; off >= 1; off >>= 1) {
    const int64_t o = __shfl_xor(end, off, 64);
    end = o > end ? o : end;
  }

  // the query row: channels 64 c + 16 g + 8 h + 0..7 of MFMA step (c, h)
  const T* q = static_cast<const T*>(a.q) + (r0 + tok) * a.ldq + (int64_t)qh * D;
  float qf[NC][16];
  float qm = 0.0f;
#pragma unroll
  for (int c = 0; c < NC; ++c)
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      qf[c][e] = live ? to_f32(q[64 * c + 16 * g + e]) : 0.0f;
      qm = amax_keep(qm, qf[c][e]);
    }
  qm = amax_keep(qm, __shfl_xor(qm, 16, 64));
  qm = amax_keep(qm, __shfl_xor(qm, 32, 64));
  int qe = 0;
  if (qm > 0.0f && qm < __builtin_inff()) qe = ilogbf(qm);
  h8 qa[NC][2];
#pragma unroll
  for (int c = 0; c < NC; ++c)
#pragma unroll
    for (int e = 0; e < 16; ++e) qa[c][e >> 3][e & 7] = (_Float16)ldexpf(qf[c][e], -qe);
  const float qscale = ldexpf(a.scale * kLog2e, qe);

  float m = -__builtin_inff(), M = m, L = 0.0f;
  fl4 o[ND];
#pragma unroll
  for (int d = 0; d < ND; ++d) o[d] = fl4{0, 0, 0, 0};

  const int32_t* table = a.table + (int64_t)s * a.table_ld;
  const int64_t page_bytes = (int64_t)P * D;
  for (int64_t t0 = (int64_t)wave * 64; t0 < end; t0 += 256) {
    // the page of a 16-token run; runs past the end read the tile's first page (their scores are masked)
    const int64_t tv = t0 + 16 * g;              // this lane's tokens
    const int64_t tk = t0 + 16 * (r >> 2);       // the tokens of this lane's key rows
    int32_t pv = table[(tv < end ? tv : t0) / P];
    int32_t pk = table[(tk < end ? tk : t0) / P];
    const bool pv_ok = pv >= 0 && pv < a.c.n_pages;
    if (!pv_ok) pv = 0;
    if (!(pk >= 0 && pk < a.c.n_pages)) pk = 0;
    const int64_t bv = (int64_t)pv * a.c.kv_heads + head, bk = (int64_t)pk * a.c.kv_heads + head;
    // how many of the lane's 16 tokens are seen
    const int64_t left = pv_ok ? lim - tv : 0;
    const int n_seen = left < 0 ? 0 : left > 16 ? 16 : (int)left;
    const float sk = a.c.k_scale[bv] * qscale, sv = a.c.v_scale[bv];
    const int8_t* kb = a.c.k + bk * page_bytes + (int64_t)((tk < end ? tk : t0) % P + (r & 3)) * D + 16 * g;
    fl4 sc[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      sc[j] = fl4{0, 0, 0, 0};
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        const u32x4_t w = *reinterpret_cast<const u32x4_t*>(kb + (int64_t)(4 * j) * D + 64 * c);
        sc[j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(codes_to_f16x8(w[0], w[1]), qa[c][0], sc[j], 0, 0, 0);
        sc[j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(codes_to_f16x8(w[2], w[3]), qa[c][1], sc[j], 0, 0, 0);
      }
    }
    float p[16];
    float run = -__builtin_inff();
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      p[e] = e < n_seen ? sc[e >> 2][e & 3] * sk : -__builtin_inff();
      run = fmaxf(run, p[e]);
    }
    const Softmax w = softmax_step(run, sv, n_seen > 0, m, M);
    float l = 0.0f;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      p[e] = __builtin_amdgcn_exp2f(p[e] + w.off);
      l += p[e];
    }
    L = L * w.alpha_l + l * w.f;
    h8 ph[2];
#pragma unroll
    for (int e = 0; e < 16; ++e) ph[e >> 3][e & 7] = (_Float16)(w.quiet ? 0.0f : p[e]);
    const int8_t* vb = a.c.v + bv * page_bytes + (int64_t)r * P + (tv < end ? tv : t0) % P;
#pragma unroll
    for (int d = 0; d < ND; ++d) {
      const u32x4_t x = *reinterpret_cast<const u32x4_t*>(vb + (int64_t)(16 * d) * P);
      fl4 acc = o[d] * w.alpha_o;
      acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(codes_to_f16x8(x[0], x[1]), ph[0], acc, 0, 0, 0);
      o[d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(codes_to_f16x8(x[2], x[3]), ph[1], acc, 0, 0, 0);
    }
  }
  L = sum_over_groups(L);
  if (g == 0) {
    sh_m[wave][r] = m;
    sh_M[wave][r] = M;
    sh_l[wave][r] = L;
  }
#pragma unroll
  for (int d = 0; d < ND; ++d) *reinterpret_cast<fl4*>(&sh_o[wave][r][16 * d + 4 * g]) = o[d];
  __syncthreads();
  for (int i = threadIdx.x; i < 16 * D; i += 256) {
    const int row = i / D, d = i - row * D;
    const int64_t RR = qt * 16 + row;
    if (RR >= n_new * G) continue;
    float mj = -__builtin_inff(), Mj = mj;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      mj = fmaxf(mj, sh_m[w][row]);
      Mj = fmaxf(Mj, sh_M[w][row]);
    }
    mj = finite_or_zero(mj);
    Mj = finite_or_zero(Mj);
    float l = 0.0f, y = 0.0f;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      l += __builtin_amdgcn_exp2f(sh_m[w][row] - mj) * sh_l[w][row];
      y += __builtin_amdgcn_exp2f(sh_M[w][row] - Mj) * sh_o[w][row][d];
    }
    y = l == 0.0f ? 0.0f : y / l * __builtin_amdgcn_exp2f(Mj - mj);
    const int64_t tk = RR / G;
    static_cast<T*>(a.out)[(r0 + tk) * a.ldo + (int64_t)(head * G + (RR - tk * G)) * D + d] = (T)y;
  }
}

template <typename T, int D>
hipError_t launch_d(const AttentionArgs& a, hipStream_t st) {
  const int64_t tiles_q = (a.max_new * (a.q_heads / a.c.kv_heads) + 15) / 16;
  const int64_t grid = (int64_t)a.n_seq * tiles_q * a.c.kv_heads;
  if (grid > 0x7FFFFFFF) return hipErrorInvalidValue;
  hipLaunchKernelGGL((k_kv_attention_rows<T, D>), dim3((unsigned)grid), dim3(256), 0, st, a, tiles_q);
  return hipGetLastError();
}

template <typename T>
hipError_t launch(const AttentionArgs& a, hipStream_t st) {
  if (a.c.head_dim == 64) return launch_d<T, 64>(a, st);
  if (a.c.head_dim == 128) return launch_d<T, 128>(a, st);
  return launch_d<T, 256>(a, st);
}

}  // namespace

size_t kv_attention_ws_bytes(const AttentionArgs&) { return 0; }

hipError_t launch_kv_attention(const AttentionArgs& a, void*, hipStream_t st) {
  if (a.n_rows < 1 || a.max_new < 1) return hipSuccess;
  return a.dtype == AWSRC_DTYPE_BF16 ? launch<__bf16>(a, st) : launch<_Float16>(a, st);
}

}  // namespace awsrc
