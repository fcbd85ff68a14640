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
  bool whole;  // every row turns by Turn
};

// Eight adjacent values; `wide`: they lie on 16 bytes.
template <typename T>
__device__ __forceinline__ void load8(const T* __restrict__ x, bool wide, float (&v)[8]) {
  awsrc::load8(x, 8, wide, v);
}
template <typename T>
__device__ __forceinline__ void store8(T* __restrict__ x, bool wide, const float (&v)[8]) {
  if (wide) {
    store_vec8(x, v);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = (T)v[e];
  }
}

// Channels d .. d + 7 (d a multiple of 8) of a rotated row; `wide`: the row lies on 16 bytes.
template <typename T>
__device__ __forceinline__ void rotated8(const T* __restrict__ x, int d, int64_t pos, const Rotary& r, bool wide, float (&y)[8]) {
  load8(x + d, wide, y);
  if (d >= 2 * r.half) return;
  const bool in = pos >= 0 && pos < r.len;
  const float* cp = r.cos + (in ? pos : 0) * r.half;
  const float* sp = r.sin + (in ? pos : 0) * r.half;
  const float nan = __builtin_nanf("");
  if (!r.interleaved && r.half % 8 == 0) {  // all eight in one half, their mates in eight adjacent places
    const bool second = d >= r.half;
    const int i = second ? d - r.half : d;
    float w[8], c[8], s[8];
    load8(x + (second ? i : i + r.half), wide, w);
    const bool four = ((reinterpret_cast<uintptr_t>(cp) | reinterpret_cast<uintptr_t>(sp)) & 15) == 0;
    if (in && four) {
#pragma unroll
      for (int e = 0; e < 8; e += 4) {
        const float4 a = *reinterpret_cast<const float4*>(cp + i + e), b = *reinterpret_cast<const float4*>(sp + i + e);
        c[e] = a.x; c[e + 1] = a.y; c[e + 2] = a.z; c[e + 3] = a.w;
        s[e] = b.x; s[e + 1] = b.y; s[e + 2] = b.z; s[e + 3] = b.w;
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        c[e] = in ? cp[i + e] : nan;
        s[e] = in ? sp[i + e] : nan;
      }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = second ? y[e] * c[e] + w[e] * s[e] : y[e] * c[e] - w[e] * s[e];
    return;
  }
  float own[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) own[e] = y[e];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const int ch = d + e;
    if (ch >= 2 * r.half) continue;
    const int i = r.interleaved ? ch >> 1 : (ch < r.half ? ch : ch - r.half);
    const bool second = r.interleaved ? (ch & 1) : ch >= r.half;
    const float w = to_f32(x[r.interleaved ? ch ^ 1 : (second ? ch - r.half : ch + r.half)]);
    const float c = in ? cp[i] : nan, s = in ? sp[i] : nan;
    y[e] = second ? own[e] * c + w * s : own[e] * c - w * s;
  }
}

// Channels i .. i + 7 and their mates half a row on, of a row rotated whole
// (rot = head_dim, halves, everything on 16 bytes).
struct Turn {
  float c[8], s[8];
  __device__ __forceinline__ void fetch(const Rotary& r, int64_t pos, int i) {
    const bool in = pos >= 0 && pos < r.len;
    const float4* cp = reinterpret_cast<const float4*>(r.cos + (in ? pos : 0) * r.half + i);
    const float4* sp = reinterpret_cast<const float4*>(r.sin + (in ? pos : 0) * r.half + i);
    const float nan = __builtin_nanf("");
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const float4 a = cp[e], b = sp[e];
      c[4 * e] = in ? a.x : nan; c[4 * e + 1] = in ? a.y : nan; c[4 * e + 2] = in ? a.z : nan; c[4 * e + 3] = in ? a.w : nan;
      s[4 * e] = in ? b.x : nan; s[4 * e + 1] = in ? b.y : nan; s[4 * e + 2] = in ? b.z : nan; s[4 * e + 3] = in ? b.w : nan;
    }
  }
  __device__ __forceinline__ void apply(float (&lo)[8], float (&hi)[8]) const {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float a = lo[e], b = hi[e];
      lo[e] = a * c[e] - b * s[e];
      hi[e] = b * c[e] + a * s[e];
    }
  }
};

// The sequence of packed row i: the last s with cu[s] <= i, or -1 outside the
// rows; a wavefront looks at 64 starts at a time.
__device__ __forceinline__ int find_seq(const int32_t* __restrict__ cu, int n_seq, int64_t i) {
  const int lane = threadIdx.x & 63;
  if (i < cu[0] || i >= cu[n_seq]) return -1;
  int lo = 0, n = n_seq;  // the answer lies in [lo, lo + n)
  while (n > 1) {
    const int step = (n + 63) / 64, at = lo + (lane + 1) * step;
    const uint64_t below = __ballot((lane + 1) * step < n && cu[at] <= i);
    const int k = __popcll(below);
    n = n - k * step < step ? n - k * step : step;
    lo += k * step;
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
  int p0, lo, hi;
  int64_t row0;
  int32_t page;  // negative where there is none
};
constexpr int kMaxTokens = 1 << 30;  // longer sequences take no part
__device__ __forceinline__ bool span_of(const int32_t* __restrict__ cu, const int32_t* __restrict__ kv_len,
                                        const int32_t* __restrict__ table, int64_t table_ld, int64_t n_pages, int64_t n_rows,
                                        int T, int s, int j, Span* o) {
  const int r0 = cu[s], r1 = cu[s + 1], len = kv_len[s];
  if (r0 < 0 || r1 <= r0 || r1 > n_rows || len < 0 || len > kMaxTokens) return false;
  const int64_t first = (int64_t)len - (r1 - r0);  // position of row r0; below 0 where a call brings more rows than tokens
  const int start = first < 0 ? 0 : (int)first;
  const int shift = __builtin_ctz(T);
  const int slot = (start >> shift) + j;
  if (slot > len >> shift) return false;
  o->p0 = slot << shift;
  o->lo = start > o->p0 ? start : o->p0;
  o->hi = len < o->p0 + T ? len : o->p0 + T;
  if (o->lo >= o->hi) return false;
  o->row0 = r0 + (o->lo - first);
  o->page = slot < table_ld ? table[(int64_t)s * table_ld + slot] : -1;
  if (o->page >= n_pages) o->page = -1;
  return true;
}

// What a thread holds of a block: four pieces of eight channels per item.  Of
// keys, an item is two times a piece and its mate half a row on.  Of values, an item is eight channels of four adjacent tokens
// (one word of each channel's row of codes); neighbouring threads take
// neighbouring words, so that a wavefront's accesses are runs of at least 16
// (pages of 16) to 64 bytes on both sides.
template <bool VALUES>
struct Place {
  int D, P;
  __device__ __forceinline__ bool at(int item, int j, int& token, int& d) const {
    if constexpr (VALUES) {
      const int x = item * 256 + threadIdx.x, shift = __builtin_ctz(P) - 2;
      token = (x & ((1 << shift) - 1)) * 4 + j;
      d = (x >> shift) * 8;
      return d < D;
    } else {
      const int x = (item * 2 + (j >> 1)) * 256 + threadIdx.x, shift = __builtin_ctz(D) - 4;
      token = x >> shift;
      d = (x & ((1 << shift) - 1)) * 8 + (j & 1) * (D >> 1);
      return token < P;
    }
  }
};

__device__ __forceinline__ uint32_t byte_at(uint32_t w, int j, int code) {
  return (w & ~(255u << (8 * j))) | (uint32_t)(code & 255) << (8 * j);
}
__device__ __forceinline__ int code_at(uint32_t w, int j) { return (int)(int8_t)(w >> (8 * j)); }

template <typename T, int NI, bool VALUES>
__device__ __forceinline__ void append_block(const AppendArgs& a, const Span& sp, int head, const Rotary& rot, bool wide) {
  const int D = a.c.head_dim, P = a.c.page_tokens;
  const int64_t ld = VALUES ? a.ldv : a.ldk;
  const T* x = static_cast<const T*>(VALUES ? a.v : a.k) + sp.row0 * ld + (int64_t)head * D;
  const int at = (int)(sp.lo - sp.p0), end = (int)(sp.hi - sp.p0);  // slots of the new tokens
  const int64_t block = (int64_t)sp.page * a.c.kv_heads + head;
  int8_t* codes = (VALUES ? a.c.v : a.c.k) + block * P * D;
  float* scale = (VALUES ? a.c.v_scale : a.c.k_scale) + block;
  const float was = at == 0 ? 0.0f : *scale;
  const Place<VALUES> place{D, P};

  float v[NI * 4][8];
  float m = 0.0f;
#pragma unroll
  for (int i = 0; i < NI; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      int t, d;
      if (!place.at(i, j, t, d) || t < at || t >= end) continue;
      const T* row = x + (t - at) * ld;
      if (VALUES || rot.whole) load8(row + d, wide, v[i * 4 + j]);
      else rotated8(row, d, sp.p0 + t, rot, wide, v[i * 4 + j]);
    }
  if constexpr (!VALUES) {
    if (rot.whole) {
#pragma unroll
      for (int i = 0; i < NI; ++i)
#pragma unroll
        for (int j = 0; j < 4; j += 2) {
          int t, d;
          if (!place.at(i, j, t, d) || t < at || t >= end) continue;
          Turn turn;
          turn.fetch(rot, sp.p0 + t, d);
          turn.apply(v[i * 4 + j], v[i * 4 + j + 1]);
        }
    }
  }
#pragma unroll
  for (int i = 0; i < NI; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      int t, d;
      if (!place.at(i, j, t, d) || t < at || t >= end) continue;
#pragma unroll
      for (int e = 0; e < 8; ++e) m = amax_keep(m, v[i * 4 + j][e]);
    }
  const float fresh = scale_of_amax(block_amax(m));
  const float now = (fresh > was || fresh != fresh) ? fresh : was;
  const float inv = inverse_scale(now);
  const bool grew = now > was && at > 0;
  const float ratio = was * inv;
  if (threadIdx.x == 0) *scale = now;  // (every thread read the old one before block_amax's barriers)
#pragma unroll
  for (int i = 0; i < NI; ++i) {
    if constexpr (VALUES) {
      int t, d;
      if (!place.at(i, 0, t, d)) continue;
      // words without a new token, or an old one to round again, stay
      if (t >= end || t + 4 <= (grew ? 0 : at)) continue;
      const bool keeps = t < at || t + 4 > end;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        uint32_t* word = reinterpret_cast<uint32_t*>(codes + (int64_t)(d + e) * P + t);
        uint32_t w = keeps ? *word : 0u;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if (t + j < at) w = grew ? byte_at(w, j, code_of((float)code_at(w, j), ratio)) : w;
          else if (t + j < end) w = byte_at(w, j, code_of(v[i * 4 + j][e], inv));
        }
        *word = w;
      }
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        int t, d;
        if (!place.at(i, j, t, d) || t >= end || (t < at && !grew)) continue;
        uint2* words = reinterpret_cast<uint2*>(codes + t * D + d);
        uint32_t w[2] = {0, 0};
        if (t < at) {
          const uint2 old = *words;
          w[0] = old.x;
          w[1] = old.y;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int c = t < at ? code_of((float)code_at(w[e >> 2], e & 3), ratio) : code_of(v[i * 4 + j][e], inv);
          w[e >> 2] = byte_at(w[e >> 2], e & 3, c);
        }
        *words = make_uint2(w[0], w[1]);
      }
    }
  }
}

// Workgroup b of those for keys and values: which of them, which head, and which
// of the n_seq * per_seq pages.
struct Work {
  int slot, head;
  bool values;
};
__device__ __forceinline__ Work work_of(uint32_t b, int heads) {
  const int slot = (int)(b >> 1) / heads;
  return {slot, (int)(b >> 1) - slot * heads, (bool)(b & 1)};
}

// Workgroups [0, n_blocks): keys and values; the rest: queries, a row a wavefront.
// Bound by bytes where tokens are many (8563 of a 32B layer: 46 us, 5.0 TB/s, a copy's rate), else by the chain of
// loads page, old scale, codes (a token each of 48 sequences of a 3B layer: 6.9 us).
template <typename T, int NI>
__global__ __launch_bounds__(256) void k_kv_append(AppendArgs a, int n_blocks, int per_seq, bool wide_kv, bool wide_q,
                                                   bool whole) {
  const Rotary rot{a.cos, a.sin, a.rope_len, a.rot / 2, a.interleaved, whole};
  const uint32_t b = workgroup<256>();
  if (b < (uint32_t)n_blocks) {
    const Work w = work_of(b, a.c.kv_heads);
    const int s = w.slot / per_seq;
    Span sp;
    if (!span_of(a.cu, a.kv_len, a.table, a.table_ld, a.c.n_pages, a.n_rows, a.c.page_tokens, s, w.slot - s * per_seq, &sp) ||
        sp.page < 0)
      return;
    if (w.values) append_block<T, NI, true>(a, sp, w.head, rot, wide_kv);
    else append_block<T, NI, false>(a, sp, w.head, rot, wide_kv);
    return;
  }
  const int64_t row = ((int64_t)b - n_blocks) * 4 + (threadIdx.x >> 6);
  if (!a.q || row >= a.n_rows) return;
  const int s = find_seq(a.cu, a.n_seq, row);
  if (s < 0) return;
  const int64_t pos = (int64_t)a.kv_len[s] - (a.cu[s + 1] - row);
  const int D = a.c.head_dim, lane = threadIdx.x & 63;
  const T* q = static_cast<const T*>(a.q) + row * a.ldq;
  T* out = static_cast<T*>(a.q_out) + row * a.ldqo;
  if (whole) {  // a lane turns the same channels of every head
    const int shift = __builtin_ctz(D) - 4, i = (lane & ((1 << shift) - 1)) * 8;
    Turn turn;
    turn.fetch(rot, pos, i);
    for (int h = lane >> shift; h < a.q_heads; h += 64 >> shift) {
      float lo[8], hi[8];
      load8(q + h * D + i, true, lo);
      load8(q + h * D + i + D / 2, true, hi);
      turn.apply(lo, hi);
      store8(out + h * D + i, true, lo);
      store8(out + h * D + i + D / 2, true, hi);
    }
    return;
  }
  const int per = D >> 3;
  for (int i = lane; i < a.q_heads * per; i += 64) {
    const int h = i / per, d = (i - h * per) * 8;
    float y[8];
    rotated8(q + h * D, d, pos, rot, wide_q, y);
    store8(out + h * D + d, wide_q, y);
  }
}

// Values lie turned in a page: their codes go through LDS (rows of P + 4 bytes,
// so that no two of a wavefront's words share a bank), from where a thread takes
// eight channels of four tokens; eight threads side by side take 64 channels of
// the same tokens, for stores of whole lines.
template <typename T, int NI, bool VALUES>
__device__ __forceinline__ void read_block(const ReadArgs& a, const Span& sp, int head, bool wide, char* lds) {
  const int D = a.c.head_dim, P = a.c.page_tokens;
  const bool there = sp.page >= 0;
  const int64_t block = (int64_t)(there ? sp.page : 0) * a.c.kv_heads + head;
  const int8_t* codes = (VALUES ? a.c.v : a.c.k) + block * P * D;
  const float sc = there ? (VALUES ? a.c.v_scale : a.c.k_scale)[block] : __builtin_nanf("");
  T* out = static_cast<T*>(VALUES ? a.v_out : a.k_out) + (sp.row0 * a.c.kv_heads + head) * D;
  const int at = (int)(sp.lo - sp.p0), end = (int)(sp.hi - sp.p0);
  if constexpr (VALUES) {
    const int shift = __builtin_ctz(P) - 4;
#pragma unroll
    for (int i = 0; i < 2 * NI; ++i) {
      const int x = i * 256 + threadIdx.x, d = x >> shift, t = (x & ((1 << shift) - 1)) * 16;
      if (d >= D || t >= end || t + 16 <= at) continue;
      const uint4 w = *reinterpret_cast<const uint4*>(codes + d * P + t);
      uint32_t* o = reinterpret_cast<uint32_t*>(lds + d * (P + 4) + t);
      o[0] = w.x; o[1] = w.y; o[2] = w.z; o[3] = w.w;
    }
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < NI; ++i) {
    uint32_t w[8];
    int vt = 0, vd = 0;
    if constexpr (VALUES) {
      const int x = i * 256 + threadIdx.x, shift = __builtin_ctz(P) - 2;
      vt = ((x >> 3) & ((1 << shift) - 1)) * 4;
      vd = ((x >> 3 >> shift) * 8 + (x & 7)) * 8;
      if (vd >= D || vt >= end || vt + 4 <= at) continue;
#pragma unroll
      for (int e = 0; e < 8; ++e) w[e] = *reinterpret_cast<const uint32_t*>(lds + (vd + e) * (P + 4) + vt);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      int t = vt + j, d = vd;
      if constexpr (!VALUES) {
        const int x = (i * 4 + j) * 256 + threadIdx.x, shift = __builtin_ctz(D) - 3;
        t = x >> shift;
        d = (x & ((1 << shift) - 1)) * 8;
      }
      if (t < at || t >= end) continue;
      float y[8];
      if constexpr (VALUES) {
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = (float)code_at(w[e], j) * sc;
      } else {
        const uint2 x = *reinterpret_cast<const uint2*>(codes + t * D + d);
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = (float)code_at(e < 4 ? x.x : x.y, e & 3) * sc;
      }
      store8(out + (int64_t)(t - at) * a.c.kv_heads * D + d, wide, y);
    }
  }
}

// Codes times scales, dense.  The same 8563 tokens: 10.5 us, 5.0 TB/s; 48 short ends of pages 4.4 us.
template <typename T, int NI>
__global__ __launch_bounds__(256) void k_kv_read(ReadArgs a, int per_seq, bool wide) {
  extern __shared__ __attribute__((aligned(16))) char lds[];
  const Work w = work_of(workgroup<256>(), a.c.kv_heads);
  const int s = w.slot / per_seq;
  if (s >= a.n_seq) return;
  Span sp;
  if (!span_of(a.cu, a.kv_len, a.table, a.table_ld, a.c.n_pages, a.n_rows, a.c.page_tokens, s, w.slot - s * per_seq, &sp))
    return;
  if (w.values) read_block<T, NI, true>(a, sp, w.head, wide, lds);
  else read_block<T, NI, false>(a, sp, w.head, wide, lds);
}

// Pages that n rows can touch from any starting position.
int64_t pages_touched(int64_t n, int T) { return n < 1 ? 0 : (n + T - 2) / T + 1; }

bool on16(const void* p, int64_t ld, int64_t size) { return ((reinterpret_cast<uintptr_t>(p) | (uintptr_t)(ld * size)) & 15) == 0; }

template <typename T, int NI>
hipError_t launch_append(const AppendArgs& a, int64_t grid, int64_t n_blocks, int64_t per_seq, hipStream_t st) {
  const bool kv = on16(a.k, a.ldk, sizeof(T)) && on16(a.v, a.ldv, sizeof(T));
  const bool q = on16(a.q, a.ldq, sizeof(T)) && on16(a.q_out, a.ldqo, sizeof(T));
  const bool whole = kv && (!a.q || q) && a.rot == a.c.head_dim && !a.interleaved && on16(a.cos, 0, 0) && on16(a.sin, 0, 0) && a.rope_len > 0;
  hipLaunchKernelGGL((k_kv_append<T, NI>), grid_of<256>(grid), dim3(256), 0, st, a, (int)n_blocks, (int)per_seq, kv, q, whole);
  return hipGetLastError();
}
template <typename T, int NI>
hipError_t launch_read(const ReadArgs& a, int64_t grid, int64_t per_seq, hipStream_t st) {
  const bool wide = on16(a.k_out, 0, 0) && on16(a.v_out, 0, 0);  // rows are a multiple of 128 bytes apart
  hipLaunchKernelGGL((k_kv_read<T, NI>), grid_of<256>(grid), dim3(256), (size_t)a.c.head_dim * (a.c.page_tokens + 4), st, a,
                     (int)per_seq, wide);
  return hipGetLastError();
}

// Items of four pieces that a block leaves each of 256 threads.
int items_of(const awsrc_kv_cache& c) {
  const int n = c.head_dim * c.page_tokens / 8192;
  return n < 1 ? 1 : n;
}

template <typename T>
hipError_t append_t(const AppendArgs& a, int64_t grid, int64_t n_blocks, int64_t per_seq, hipStream_t st) {
  switch (items_of(a.c)) {
    case 1: return launch_append<T, 1>(a, grid, n_blocks, per_seq, st);
    case 2: return launch_append<T, 2>(a, grid, n_blocks, per_seq, st);
    default: return launch_append<T, 4>(a, grid, n_blocks, per_seq, st);
  }
}
template <typename T>
hipError_t read_t(const ReadArgs& a, int64_t grid, int64_t per_seq, hipStream_t st) {
  switch (items_of(a.c)) {
    case 1: return launch_read<T, 1>(a, grid, per_seq, st);
    case 2: return launch_read<T, 2>(a, grid, per_seq, st);
    default: return launch_read<T, 4>(a, grid, per_seq, st);
  }
}

}  // namespace

hipError_t launch_kv_append(const AppendArgs& a, hipStream_t st) {
  const int64_t per_seq = pages_touched(a.max_new, a.c.page_tokens);
  const int64_t n_blocks = 2 * a.n_seq * per_seq * a.c.kv_heads;
  const int64_t grid = n_blocks + (a.q ? (a.n_rows + 3) / 4 : 0);
  if (grid <= 0) return hipSuccess;
  if (grid > 0x7FFFFFFF) return hipErrorInvalidValue;
  if (a.dtype == AWSRC_DTYPE_F32) return append_t<float>(a, grid, n_blocks, per_seq, st);
  if (a.dtype == AWSRC_DTYPE_BF16) return append_t<__bf16>(a, grid, n_blocks, per_seq, st);
  return append_t<_Float16>(a, grid, n_blocks, per_seq, st);
}

hipError_t launch_kv_read(const ReadArgs& a, hipStream_t st) {
  const int64_t per_seq = pages_touched(a.max_rows, a.c.page_tokens);
  const int64_t grid = 2 * a.n_seq * per_seq * a.c.kv_heads;
  if (grid <= 0) return hipSuccess;
  if (grid > 0x7FFFFFFF) return hipErrorInvalidValue;
  if (a.dtype == AWSRC_DTYPE_F32) return read_t<float>(a, grid, per_seq, st);
  if (a.dtype == AWSRC_DTYPE_BF16) return read_t<__bf16>(a, grid, per_seq, st);
  return read_t<_Float16>(a, grid, per_seq, st);
}

}  // namespace awsrc
