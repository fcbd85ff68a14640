// The paged int8 cache of keys and values: appending tokens (keys rotated by
// position, queries rotated on the way) and reading tokens back.
//
// A page holds page_tokens tokens of every head, with one scale per head for
// its keys and one for its values.  Keys lie as [token][channel], values as
// [channel][token]: the attention kernel's matrix products take both in
// 16-byte runs along their sum, channels for the scores and tokens for the
// output, straight from memory.
//
// One workgroup owns the keys or the values of one (sequence, page, head):
// the largest magnitude of the page's new tokens, the page's scale (it only
// grows while the page fills, and starts anew when its first slot is
// written), the older codes rounded to it where it grew, the new codes.  No
// atomics, so that a call's result does not depend on any order.
//
// Built without FMA contraction: rotation, scale and codes are single fp32
// operations.
#include "serve_internal.h"

namespace awsrc {

namespace {

// Rotation of one position: pair (i, i + rot/2), or (2 i, 2 i + 1) where
// interleaved; channels from rot on pass through.  Positions outside the
// table rotate by NaN, which the page's scale then carries into every result.
struct Rotary {
  const float *cos, *sin;
  int64_t len;
  int half, interleaved;
};

template <typename T>
__device__ __forceinline__ float rotated(const T* __restrict__ x, int d, int64_t pos, const Rotary& r) {
  const float v = to_f32(x[d]);
  if (d >= 2 * r.half) return v;
  const int i = r.interleaved ? d >> 1 : (d < r.half ? d : d - r.half);
  const bool second = r.interleaved ? (d & 1) : d >= r.half;
  const int mate = r.interleaved ? d ^ 1 : (second ? d - r.half : d + r.half);
  const bool in = pos >= 0 && pos < r.len;
  const float c = in ? r.cos[pos * r.half + i] : __builtin_nanf("");
  const float s = in ? r.sin[pos * r.half + i] : __builtin_nanf("");
  const float w = to_f32(x[mate]);
  return second ? v * c + w * s : v * c - w * s;
}

// The sequence of packed row i: the last s with cu[s] <= i, or -1 past the last row.
__device__ __forceinline__ int find_seq(const int32_t* __restrict__ cu, int n_seq, int64_t i) {
  if (i < cu[0] || i >= cu[n_seq]) return -1;
  int lo = 0, hi = n_seq;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (cu[mid] <= i) lo = mid; else hi = mid;
  }
  return lo;
}

__device__ __forceinline__ float block_amax(float m) {
  __shared__ float part[4];
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) m = amax_keep(m, __shfl_xor(m, off, 64));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = m;
  __syncthreads();
  m = part[0];
#pragma unroll
  for (int w = 1; w < 4; ++w) m = amax_keep(m, part[w]);
  return m;
}

// Which tokens of page slot j (counted from the first touched page) are new:
// positions [lo, hi), page positions from p0; the rows of k and v start at row0 for lo.
struct Span {
  int64_t p0, lo, hi, row0;
  int32_t page;  // negative where there is none
};
__device__ __forceinline__ bool span_of(const int32_t* cu, const int32_t* kv_len, const int32_t* table, int64_t table_ld,
                                        int64_t n_pages, int64_t n_rows, int T, int s, int64_t j, Span* o) {
  int64_t r0 = cu[s], r1 = cu[s + 1];
  if (r0 < 0) return false;
  if (r1 > n_rows) r1 = n_rows;
  const int64_t len = kv_len[s];
  const int64_t first = len - (cu[s + 1] - r0);  // position of row r0; below 0 where a call brings more rows than tokens
  const int64_t start = first < 0 ? 0 : first;
  const int64_t slot = start / T + j;
  o->p0 = slot * T;
  o->lo = start > o->p0 ? start : o->p0;
  const int64_t end = len < first + (r1 - r0) ? len : first + (r1 - r0);
  o->hi = end < o->p0 + T ? end : o->p0 + T;
  if (o->lo >= o->hi) return false;
  o->row0 = r0 + (o->lo - first);
  o->page = slot < table_ld ? table[(int64_t)s * table_ld + slot] : -1;
  if (o->page >= n_pages) o->page = -1;
  return true;
}

template <typename T>
__device__ void append_block(const AppendArgs& a, const Span& sp, int head, bool values, const Rotary& rot) {
  const int D = a.c.head_dim, P = a.c.page_tokens;
  const int64_t ld = values ? a.ldv : a.ldk;
  const T* x = static_cast<const T*>(values ? a.v : a.k) + sp.row0 * ld + (int64_t)head * D;
  const int n_new = (int)(sp.hi - sp.lo), at = (int)(sp.lo - sp.p0);
  const int64_t block = (int64_t)sp.page * a.c.kv_heads + head;
  int8_t* codes = (values ? a.c.v : a.c.k) + block * P * D;
  float* scale = (values ? a.c.v_scale : a.c.k_scale) + block;

  float m = 0.0f;
  for (int i = threadIdx.x; i < n_new * D; i += 256) {
    const int t = i / D, d = i - t * D;
    m = amax_keep(m, values ? to_f32(x[t * ld + d]) : rotated(x + t * ld, d, sp.lo + t, rot));
  }
  const float fresh = scale_of_amax(block_amax(m));
  const float was = at == 0 ? 0.0f : *scale;
  const float now = (fresh > was || fresh != fresh) ? fresh : was;
  const float inv = inverse_scale(now);
  __syncthreads();  // every thread has read the old scale
  if (threadIdx.x == 0) *scale = now;
  if (now > was && at > 0) {
    const float ratio = was * inv;
    for (int i = threadIdx.x; i < at * D; i += 256) {
      const int t = i / D, d = i - t * D;
      int8_t* c = codes + (values ? (int64_t)d * P + t : (int64_t)t * D + d);
      *c = (int8_t)code_of((float)*c, ratio);
    }
  }
  for (int i = threadIdx.x; i < n_new * D; i += 256) {
    const int t = i / D, d = i - t * D;
    const float v = values ? to_f32(x[t * ld + d]) : rotated(x + t * ld, d, sp.lo + t, rot);
    codes[values ? (int64_t)d * P + at + t : (int64_t)(at + t) * D + d] = (int8_t)code_of(v, inv);
  }
}

// Workgroups [0, n_blocks): keys and values; the rest: one row of queries each.
template <typename T>
__global__ __launch_bounds__(256) void k_kv_append(AppendArgs a, int64_t n_blocks, int64_t per_seq) {
  const Rotary rot{a.cos, a.sin, a.rope_len, a.rot / 2, a.interleaved};
  int64_t b = blockIdx.x;
  if (b < n_blocks) {
    const bool values = b & 1;
    b >>= 1;
    const int head = (int)(b % a.c.kv_heads);
    b /= a.c.kv_heads;
    const int s = (int)(b / per_seq);
    Span sp;
    if (!span_of(a.cu, a.kv_len, a.table, a.table_ld, a.c.n_pages, a.n_rows, a.c.page_tokens, s, b % per_seq, &sp) || sp.page < 0) return;
    append_block<T>(a, sp, head, values, rot);
    return;
  }
  const int64_t row = b - n_blocks;
  const int s = find_seq(a.cu, a.n_seq, row);
  if (s < 0) return;
  const int64_t pos = (int64_t)a.kv_len[s] - (a.cu[s + 1] - row);
  const int D = a.c.head_dim;
  for (int i = threadIdx.x; i < a.q_heads * D; i += 256) {
    const int h = i / D, d = i - h * D;
    static_cast<T*>(a.q_out)[row * a.ldqo + i] = (T)rotated(static_cast<const T*>(a.q) + row * a.ldq + (int64_t)h * D, d, pos, rot);
  }
}

template <typename T>
__global__ __launch_bounds__(256) void k_kv_read(ReadArgs a, int64_t per_seq) {
  const int D = a.c.head_dim, P = a.c.page_tokens;
  int64_t b = blockIdx.x;
  const bool values = b & 1;
  b >>= 1;
  const int head = (int)(b % a.c.kv_heads);
  b /= a.c.kv_heads;
  const int s = (int)(b / per_seq);
  Span sp;
  if (!span_of(a.cu, a.kv_len, a.table, a.table_ld, a.c.n_pages, a.n_rows, P, s, b % per_seq, &sp)) return;
  const bool there = sp.page >= 0;
  const int64_t block = (int64_t)(there ? sp.page : 0) * a.c.kv_heads + head;
  const int8_t* codes = (values ? a.c.v : a.c.k) + block * P * D;
  const float sc = there ? (values ? a.c.v_scale : a.c.k_scale)[block] : __builtin_nanf("");
  T* out = static_cast<T*>(values ? a.v_out : a.k_out);
  const int at = (int)(sp.lo - sp.p0), n = (int)(sp.hi - sp.lo);
  for (int i = threadIdx.x; i < n * D; i += 256) {
    const int t = i / D, d = i - t * D;
    const int8_t c = codes[values ? (int64_t)d * P + at + t : (int64_t)(at + t) * D + d];
    out[((sp.row0 + t) * a.c.kv_heads + head) * D + d] = (T)((float)c * sc);
  }
}

// Pages that n rows can touch from any starting position.
int64_t pages_touched(int64_t n, int T) { return n < 1 ? 0 : (n + T - 2) / T + 1; }

}  // namespace

hipError_t launch_kv_append(const AppendArgs& a, hipStream_t st) {
  const int64_t per_seq = pages_touched(a.max_new, a.c.page_tokens);
  const int64_t n_blocks = 2 * a.n_seq * per_seq * a.c.kv_heads;
  const int64_t grid = n_blocks + (a.q ? a.n_rows : 0);
  if (grid <= 0) return hipSuccess;
  if (grid > 0x7FFFFFFF) return hipErrorInvalidValue;
  if (a.dtype == AWSRC_DTYPE_F32)
    hipLaunchKernelGGL((k_kv_append<float>), dim3((unsigned)grid), dim3(256), 0, st, a, n_blocks, per_seq);
  else if (a.dtype == AWSRC_DTYPE_BF16)
    hipLaunchKernelGGL((k_kv_append<__bf16>), dim3((unsigned)grid), dim3(256), 0, st, a, n_blocks, per_seq);
  else
    hipLaunchKernelGGL((k_kv_append<_Float16>), dim3((unsigned)grid), dim3(256), 0, st, a, n_blocks, per_seq);
  return hipGetLastError();
}

hipError_t launch_kv_read(const ReadArgs& a, hipStream_t st) {
  const int64_t per_seq = pages_touched(a.max_rows, a.c.page_tokens);
  const int64_t grid = 2 * a.n_seq * per_seq * a.c.kv_heads;
  if (grid <= 0) return hipSuccess;
  if (grid > 0x7FFFFFFF) return hipErrorInvalidValue;
  if (a.dtype == AWSRC_DTYPE_F32)
    hipLaunchKernelGGL((k_kv_read<float>), dim3((unsigned)grid), dim3(256), 0, st, a, per_seq);
  else if (a.dtype == AWSRC_DTYPE_BF16)
    hipLaunchKernelGGL((k_kv_read<__bf16>), dim3((unsigned)grid), dim3(256), 0, st, a, per_seq);
  else
    hipLaunchKernelGGL((k_kv_read<_Float16>), dim3((unsigned)grid), dim3(256), 0, st, a, per_seq);
  return hipGetLastError();
}

}  // namespace awsrc
