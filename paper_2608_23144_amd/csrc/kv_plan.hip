// The plan of a step's pages and rows, on the device.
//
// Two launches.  One workgroup scans the request slots: who is served, where
// each one's rows start, where its pages lie in the order of pages taken and in that
// of pages given back.  Then one thread a row finds its slot, position and page, and
// writes the page table where a row is the first of a page taken.  The t-th page
// taken is the t-th given back, or the free stack's (t - given)-th from the top:
// no thread waits for another, and no order depends on a run.  Taken pages and
// pages given back belong to different rows of the table, and the stack is
// written only where more is given back than taken, when nothing is taken from it.
#include "serve_internal.h"

namespace awsrc {

namespace {

// What the scan leaves for the rows: first the header, then one entry per slot.
struct PlanHead {
  int64_t n_free, given;
  int64_t taken;
  int64_t rows;
};
struct PlanSlot {
  int32_t take, give;  // places of its first page among those taken, and among those given back
  int32_t held, want;  // pages before and after
};

struct Lengths {
  int64_t keep, fresh, held, want;
};

__device__ __forceinline__ Lengths lengths_of(const PlanArgs& a, int s) {
  const int P = a.pool.page_tokens;
  const int64_t most = a.table_ld * P;
  int64_t kv = a.kv_len[s], keep = a.keep[s], fresh = a.new_len[s];
  kv = kv < 0 ? 0 : kv < most ? kv : most;
  keep = keep < 0 ? 0 : keep < kv ? keep : kv;
  fresh = fresh < 0 ? 0 : fresh;
  return {keep, fresh, (kv + P - 1) / P, (keep + fresh + P - 1) / P};
}

// Inclusive sums over the workgroup's threads; `total` is everyone's.
template <int W, typename T>
__device__ __forceinline__ T scan(T x, T* wave_sums, T& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const T y = __shfl_up(x, off, 64);
    if (lane >= off) x += y;
  }
  if (lane == 63) wave_sums[wave] = x;
  __syncthreads();
  T before = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < W; ++w) {
    if (w < wave) before += wave_sums[w];
    total += wave_sums[w];
  }
  __syncthreads();
  return x + before;
}

__global__ __launch_bounds__(1024) void k_plan_scan(PlanArgs a, PlanHead* head, PlanSlot* slots) {
  __shared__ int64_t sums[16];
  const int P = a.pool.page_tokens, tid = threadIdx.x;
  int64_t n_free = a.pool.n_free[0];
  n_free = n_free < 0 ? 0 : n_free < a.pool.n_pages ? n_free : a.pool.n_pages;
  // what all slots give back, before anyone is turned away
  int64_t back = 0, spare;
  for (int s = tid; s < a.n_seq; s += 1024) {
    const Lengths l = lengths_of(a, s);
    back += l.held > l.want ? l.held - l.want : 0;
  }
  scan<16>(back, sums, spare);
  spare += n_free;
  int64_t asked = 0, queued = 0, rows = 0, taken = 0, given = 0;
  for (int s0 = 0; s0 < a.n_seq; s0 += 1024) {
    const int s = s0 + tid;
    const bool live = s < a.n_seq;
    Lengths l = {0, 0, 0, 0};
    if (live) l = lengths_of(a, s);
    const int64_t need = l.want > l.held ? l.want - l.held : 0;
    int64_t all;
    const int64_t pages_so_far = asked + scan<16>(need, sums, all);
    asked += all;
    const int64_t rows_so_far = queued + scan<16>(l.fresh, sums, all);
    queued += all;
    const bool served = l.want <= a.table_ld && (need == 0 || pages_so_far <= spare) && rows_so_far <= a.max_rows;
    if (!served) {
      l.fresh = 0;
      l.want = (l.keep + P - 1) / P;
    }
    const int64_t take = l.want > l.held ? l.want - l.held : 0, give = l.held > l.want ? l.held - l.want : 0;
    const int64_t t = taken + scan<16>(take, sums, all) - take;
    taken += all;
    const int64_t g = given + scan<16>(give, sums, all) - give;
    given += all;
    const int64_t r = rows + scan<16>(l.fresh, sums, all);
    rows += all;
    if (live) {
      a.kv_out[s] = (int32_t)(l.keep + l.fresh);
      a.cu[s + 1] = (int32_t)r;
      slots[s] = {(int32_t)t, (int32_t)g, (int32_t)l.held, (int32_t)l.want};
    }
  }
  if (tid == 0) {
    a.cu[0] = 0;
    const int64_t left = n_free + given - taken;
    a.n_free_out[0] = (int32_t)(left < a.pool.n_pages ? left : a.pool.n_pages);
    *head = {n_free, given, taken, rows};
  }
}

// The j-th page given back: the last slot whose pages given back start at or before j.
__device__ __forceinline__ int32_t page_given(const PlanArgs& a, const PlanSlot* slots, int64_t j) {
  int lo = 0, hi = a.n_seq;
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (slots[mid].give <= j) lo = mid;
    else hi = mid;
  }
  return a.table[lo * a.table_ld + slots[lo].want + (j - slots[lo].give)];
}

__global__ __launch_bounds__(256) void k_plan_rows(PlanArgs a, const PlanHead* head, const PlanSlot* slots) {
  const PlanHead h = *head;
  const int P = a.pool.page_tokens;
  const int64_t first = (int64_t)blockIdx.x * 256 + threadIdx.x, step = (int64_t)gridDim.x * 256;
  for (int64_t row = first; row < a.max_rows; row += step) {
    int32_t seq = -1, pos = -1;
    int64_t slot = -1;
    if (row < h.rows) {
      int lo = 0, hi = a.n_seq;  // the last slot whose rows start at or before this one
      while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (a.cu[mid] <= row) lo = mid;
        else hi = mid;
      }
      seq = lo;
      const int32_t start = a.cu[lo];
      pos = (int32_t)(a.kv_out[lo] - (a.cu[lo + 1] - start) + (row - start));
      const PlanSlot q = slots[lo];
      const int32_t at = pos / P;
      int32_t* entry = a.table + lo * a.table_ld + at;
      int32_t page;
      if (at < q.held) {
        page = *entry;
      } else {
        const int64_t t = (int64_t)q.take + at - q.held;
        page = t < h.given ? page_given(a, slots, t) : a.pool.free_pages[h.n_free - 1 - (t - h.given)];
        if (pos % P == 0) *entry = page;
      }
      if (page >= 0 && page < a.pool.n_pages) slot = (int64_t)page * P + pos % P;
    }
    if (a.row_seq) a.row_seq[row] = seq;
    if (a.row_pos) a.row_pos[row] = pos;
    if (a.row_slot) a.row_slot[row] = slot;
  }
  for (int64_t j = h.taken + first; j < h.given; j += step) {
    const int64_t at = h.n_free + h.given - 1 - j;
    if (at < a.pool.n_pages) a.pool.free_pages[at] = page_given(a, slots, j);
  }
}

}  // namespace

size_t kv_plan_ws_bytes(int n_seq) { return n_seq ? 256 + (size_t)n_seq * sizeof(PlanSlot) : 0; }

hipError_t launch_kv_plan(const PlanArgs& a, void* ws, hipStream_t st) {
  PlanHead* head = static_cast<PlanHead*>(ws);
  PlanSlot* slots = reinterpret_cast<PlanSlot*>(static_cast<char*>(ws) + 256);
  hipLaunchKernelGGL(k_plan_scan, dim3(1), dim3(1024), 0, st, a, head, slots);
  const int64_t want = (a.max_rows + 255) / 256;
  hipLaunchKernelGGL(k_plan_rows, dim3((unsigned)(want < 64 ? 64 : want < 4096 ? want : 4096)), dim3(256), 0, st, a, head, slots);
  return hipGetLastError();
}

}  // namespace awsrc
