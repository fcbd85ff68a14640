// The plan of a step's pages and rows, on the device.
//
// One workgroup scans the request slots: who is served, where each one's rows
// start, where its pages lie in the order of pages taken and in that of pages given
// back.  Then threads find the slot, position and page of their rows, and write
// the page table where a row is the first of a page taken.  The t-th page taken
// is the t-th given back, or the free stack's (t - given)-th from the top:
// no thread waits for another, and no order depends on a run.  Taken pages and
// pages given back belong to different rows of the table, and the stack is
// written only where more is given back than taken, when nothing is taken from it.
//
// Bound by latency: a few loads that wait for one another and the scans between
// them.  Steps of at most 2048 slots and 8192 rows run in one launch of one workgroup:
// 48 sequences of up to 5 rows 5.4 us, 2048 with 2051 rows 9.4.  2048 slots with prompts, 325764
// rows: 17.4 us in two launches, 7 of them the scan by one workgroup.
#include "serve_internal.h"

namespace awsrc {

namespace {

// What the scan leaves for the rows: first the header, then one entry per slot.
struct PlanHead {
  int64_t n_free, given, taken, rows;
};
struct PlanSlot {
  int32_t held;   // pages that it has
  int32_t taken;  // the place among the pages taken that its page 0 would have
  int32_t pos;    // the position that row 0 would have
  int32_t given;  // the place in the table of page 0 of those given back, seen from its own
};
// Where the rows find it, in LDS or in memory.
struct Plan {
  const PlanSlot* slots;
  const int32_t *cu, *give;  // starts of the slots' rows, and of their pages given back
};

struct Lengths {
  int64_t keep, fresh, held, want;
};

__device__ __forceinline__ int64_t pages_of(int64_t tokens, int shift) { return (tokens + (1 << shift) - 1) >> shift; }

__device__ __forceinline__ Lengths lengths_of(int64_t kv, int64_t keep, int64_t fresh, int64_t table_ld, int shift) {
  const int64_t most = table_ld << shift;
  kv = kv < 0 ? 0 : kv < most ? kv : most;
  keep = keep < 0 ? 0 : keep < kv ? keep : kv;
  fresh = fresh < 0 ? 0 : fresh;
  return {keep, fresh, pages_of(kv, shift), pages_of(keep + fresh, shift)};
}

// The last of n places whose value is at most x (value(0) is).
template <typename F>
__device__ __forceinline__ int last_at_most(int n, int64_t x, const F& value) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (value(mid) <= x) lo = mid;
    else hi = mid;
  }
  return lo;
}

// The j-th page given back: of the last slot whose pages given back start at or before j.
__device__ __forceinline__ int32_t page_given(const PlanArgs& a, const Plan& plan, int64_t j) {
  const int s = last_at_most(a.n_seq, j, [&](int i) { return plan.give[i]; });
  return a.table[plan.slots[s].given + j];
}

// Rows row .. row + 3 of the step, and every step-th four after them.
__device__ __forceinline__ void plan_rows(const PlanArgs& a, const PlanHead& h, const Plan& plan, int64_t first, int64_t step) {
  const int shift = __builtin_ctz(a.pool.page_tokens), P = a.pool.page_tokens;
  for (int64_t row0 = first * 4; row0 < a.max_rows; row0 += step * 4) {
    int32_t seq[4], pos[4];
    int64_t slot[4];
    int s = row0 < h.rows ? last_at_most(a.n_seq, row0, [&](int i) { return plan.cu[i]; }) : 0;
    int32_t end = -1, at = -1, page = -1;
    PlanSlot q = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int64_t row = row0 + i;
      seq[i] = pos[i] = -1;
      slot[i] = -1;
      if (row >= h.rows) continue;
      if (row >= end) {  // the next slot that has rows
        if (end >= 0) do ++s;
          while (plan.cu[s + 1] <= row);
        end = plan.cu[s + 1];
        q = plan.slots[s];
        at = -1;
      }
      seq[i] = s;
      pos[i] = q.pos + (int32_t)row;
      if (pos[i] >> shift != at) {
        at = pos[i] >> shift;
        int32_t* entry = a.table + s * a.table_ld + at;
        if (at < q.held) {
          page = *entry;
        } else {
          const int64_t t = q.taken + at;
          page = t < h.given ? page_given(a, plan, t) : a.pool.free_pages[h.n_free - 1 - (t - h.given)];
          if ((pos[i] & (P - 1)) == 0) *entry = page;
        }
      }
      if (page >= 0 && page < a.pool.n_pages) slot[i] = ((int64_t)page << shift) + (pos[i] & (P - 1));
    }
    const bool four = row0 + 4 <= a.max_rows;
    typedef int32_t i4_any __attribute__((ext_vector_type(4), aligned(4)));
    typedef int64_t l2_any __attribute__((ext_vector_type(2), aligned(8)));
    if (four) {
      if (a.row_seq) *reinterpret_cast<i4_any*>(a.row_seq + row0) = i4_any{seq[0], seq[1], seq[2], seq[3]};
      if (a.row_pos) *reinterpret_cast<i4_any*>(a.row_pos + row0) = i4_any{pos[0], pos[1], pos[2], pos[3]};
      if (a.row_slot) {
        *reinterpret_cast<l2_any*>(a.row_slot + row0) = l2_any{slot[0], slot[1]};
        *reinterpret_cast<l2_any*>(a.row_slot + row0 + 2) = l2_any{slot[2], slot[3]};
      }
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (row0 + i < a.max_rows) {
          if (a.row_seq) a.row_seq[row0 + i] = seq[i];
          if (a.row_pos) a.row_pos[row0 + i] = pos[i];
          if (a.row_slot) a.row_slot[row0 + i] = slot[i];
        }
    }
  }
  // pages given back that nobody took, onto the stack
  for (int64_t j = h.taken + first; j < h.given; j += step) {
    const int64_t at = h.n_free + h.given - 1 - j;
    if (at < a.pool.n_pages) a.pool.free_pages[at] = page_given(a, plan, j);
  }
}

template <int N>
using Ints = int32_t __attribute__((ext_vector_type(N), aligned(4)));

// A thread takes I slots side by side, whose loads are on their way together.  ALONE: the rows too, for at most 64 W I slots.
template <int W, int I, bool ALONE>
__global__ __launch_bounds__(64 * W) void k_plan_scan(PlanArgs a, PlanHead* head, PlanSlot* slots, int32_t* gives) {
  constexpr int kChunk = 64 * W * I;
  __shared__ int64_t sums[3][3][W];
  __shared__ int32_t s_give[ALONE ? kChunk : 1];
  __shared__ PlanSlot s_slots[ALONE ? kChunk : 1];
  __shared__ int32_t s_cu[ALONE ? kChunk + 1 : 1];
  const int shift = __builtin_ctz(a.pool.page_tokens), tid = threadIdx.x;
  int64_t n_free = a.pool.n_free[0];
  n_free = n_free < 0 ? 0 : n_free < a.pool.n_pages ? n_free : a.pool.n_pages;
  Lengths l[I];
  const auto read = [&](int s0) {
    Ints<I> kv = {}, keep = {}, fresh = {};
    const int s = s0 + tid * I;
    if (s + I <= a.n_seq) {
      kv = *reinterpret_cast<const Ints<I>*>(a.kv_len + s);
      keep = *reinterpret_cast<const Ints<I>*>(a.keep + s);
      fresh = *reinterpret_cast<const Ints<I>*>(a.new_len + s);
    } else {
#pragma unroll
      for (int i = 0; i < I; ++i)
        if (s + i < a.n_seq) {
          kv[i] = a.kv_len[s + i];
          keep[i] = a.keep[s + i];
          fresh[i] = a.new_len[s + i];
        }
    }
#pragma unroll
    for (int i = 0; i < I; ++i) l[i] = lengths_of(kv[i], keep[i], fresh[i], a.table_ld, shift);
  };
  // what all slots give back, before anyone is turned away
  int64_t back[1] = {0}, spare[1];
  for (int s0 = 0; s0 < a.n_seq; s0 += kChunk) {
    read(s0);
#pragma unroll
    for (int i = 0; i < I; ++i) back[0] += l[i].held > l[i].want ? l[i].held - l[i].want : 0;
  }
  scan_workgroup<W, 1>(back, spare, sums[0]);
  spare[0] += n_free;
  int64_t asked = 0, queued = 0, rows = 0, taken = 0, given = 0;
  for (int s0 = 0; s0 < a.n_seq; s0 += kChunk) {
    if (a.n_seq > kChunk) read(s0);
    int64_t x[2] = {0, 0}, all[2];
#pragma unroll
    for (int i = 0; i < I; ++i) {
      x[0] += l[i].want > l[i].held ? l[i].want - l[i].held : 0;
      x[1] += l[i].fresh;
    }
    const int64_t need_here = x[0], fresh_here = x[1];
    scan_workgroup<W, 2>(x, all, sums[1]);
    int64_t pages = asked + x[0] - need_here, queue = queued + x[1] - fresh_here;
    asked += all[0];
    queued += all[1];
    int64_t y[3] = {0, 0, 0}, sum[3];
#pragma unroll
    for (int i = 0; i < I; ++i) {
      const int64_t need = l[i].want > l[i].held ? l[i].want - l[i].held : 0;
      pages += need;
      queue += l[i].fresh;
      if (!(l[i].want <= a.table_ld && (need == 0 || pages <= spare[0]) && queue <= a.max_rows)) {
        l[i].fresh = 0;
        l[i].want = pages_of(l[i].keep, shift);
      }
      y[0] += l[i].want > l[i].held ? l[i].want - l[i].held : 0;
      y[1] += l[i].held > l[i].want ? l[i].held - l[i].want : 0;
      y[2] += l[i].fresh;
    }
    const int64_t take_here = y[0], give_here = y[1], rows_here = y[2];
    scan_workgroup<W, 3>(y, sum, sums[2]);
    int64_t take = taken + y[0] - take_here, give = given + y[1] - give_here, row = rows + y[2] - rows_here;
    Ints<I> kv_out, cu, starts;
    const bool whole = s0 + tid * I + I <= a.n_seq;
#pragma unroll
    for (int i = 0; i < I; ++i) {
      const int s = s0 + tid * I + i;
      const PlanSlot q = {(int32_t)l[i].held, (int32_t)(take - l[i].held), (int32_t)(l[i].keep - row),
                          (int32_t)(s * a.table_ld + l[i].want - give)};
      kv_out[i] = (int32_t)(l[i].keep + l[i].fresh);
      cu[i] = (int32_t)(row + l[i].fresh);
      starts[i] = (int32_t)give;
      if (s < a.n_seq) {
        if constexpr (ALONE) {
          s_slots[s] = q;
          s_give[s] = starts[i];
          s_cu[s + 1] = cu[i];
        } else {
          slots[s] = q;
          if (!whole) gives[s] = starts[i];
        }
        if (!whole) {
          a.kv_out[s] = kv_out[i];
          a.cu[s + 1] = cu[i];
        }
      }
      take += l[i].want > l[i].held ? l[i].want - l[i].held : 0;
      give += l[i].held > l[i].want ? l[i].held - l[i].want : 0;
      row += l[i].fresh;
    }
    if (whole) {
      const int s = s0 + tid * I;
      *reinterpret_cast<Ints<I>*>(a.kv_out + s) = kv_out;
      *reinterpret_cast<Ints<I>*>(a.cu + s + 1) = cu;
      if (!ALONE) *reinterpret_cast<Ints<I>*>(gives + s) = starts;
    }
    taken += sum[0];
    given += sum[1];
    rows += sum[2];
    if (a.n_seq > kChunk) __syncthreads();  // (the sums are written again)
  }
  const PlanHead h = {n_free, given, taken, rows};
  if (tid == 0) {
    a.cu[0] = 0;
    if (ALONE) s_cu[0] = 0;
    const int64_t left = n_free + given - taken;
    a.n_free_out[0] = (int32_t)(left < a.pool.n_pages ? left : a.pool.n_pages);
    if (!ALONE) *head = h;
  }
  if constexpr (ALONE) {
    __syncthreads();
    plan_rows(a, h, Plan{s_slots, s_cu, s_give}, tid, 64 * W);
  }
}

constexpr int kStaged = 2048;  // slots whose starts a workgroup keeps in LDS

__global__ __launch_bounds__(256) void k_plan_rows(PlanArgs a, const PlanHead* head, const PlanSlot* slots, const int32_t* gives) {
  __shared__ int32_t s_cu[kStaged + 1], s_give[kStaged];
  const bool staged = a.n_seq <= kStaged;
  const PlanHead h = *head;
  if (staged) {
    int32_t c[kStaged / 256], g[kStaged / 256];
#pragma unroll
    for (int i = 0; i < kStaged / 256; ++i) {
      const int s = i * 256 + threadIdx.x;
      c[i] = s < a.n_seq ? a.cu[s + 1] : 0;
      g[i] = s < a.n_seq ? gives[s] : 0;
    }
#pragma unroll
    for (int i = 0; i < kStaged / 256; ++i) {
      s_cu[i * 256 + threadIdx.x + 1] = c[i];
      s_give[i * 256 + threadIdx.x] = g[i];
    }
    if (threadIdx.x == 0) s_cu[0] = 0;
  }
  __syncthreads();
  const int64_t first = (int64_t)blockIdx.x * 256 + threadIdx.x, step = (int64_t)gridDim.x * 256;
  if (staged) plan_rows(a, h, Plan{slots, s_cu, s_give}, first, step);
  else plan_rows(a, h, Plan{slots, a.cu, gives}, first, step);
}

}  // namespace

// One workgroup does it all where its threads have a few slots and rows each (in one launch and in two: 300 slots with 1499
// rows 9.2 and 12.5 us, 1000 with 5001 12.4 and 14.2, 2048 with 6147 13.1 and 14.4; 1000 with 8998 16.1 and 14.3, but a launch
// costs the host 3).
static bool plan_alone(int n_seq, int64_t max_rows) { return n_seq <= 2048 && max_rows <= 8192; }

size_t kv_plan_ws_bytes(int n_seq, int64_t max_rows) {
  return !plan_alone(n_seq, max_rows) ? 256 + (size_t)n_seq * (sizeof(PlanSlot) + 4) : 0;
}

template <int W, int I>
static hipError_t launch_alone(const PlanArgs& a, hipStream_t st) {
  hipLaunchKernelGGL((k_plan_scan<W, I, true>), dim3(1), dim3(64 * W), 0, st, a, (PlanHead*)nullptr, (PlanSlot*)nullptr, (int32_t*)nullptr);
  return hipGetLastError();
}

hipError_t launch_kv_plan(const PlanArgs& a, void* ws, hipStream_t st) {
  if (plan_alone(a.n_seq, a.max_rows)) {
    // (200 slots with 994 rows by four wavefronts 7.0 us; with 1783 10.0, with 3371 by sixteen 9.1)
    if (a.n_seq <= 256 && a.max_rows <= 1024) return launch_alone<4, 1>(a, st);
    return a.n_seq <= 1024 ? launch_alone<16, 1>(a, st) : launch_alone<16, 2>(a, st);
  }
  PlanHead* head = static_cast<PlanHead*>(ws);
  PlanSlot* slots = reinterpret_cast<PlanSlot*>(static_cast<char*>(ws) + 256);
  int32_t* gives = reinterpret_cast<int32_t*>(slots + a.n_seq);
  if (a.n_seq <= 256) hipLaunchKernelGGL((k_plan_scan<4, 1, false>), dim3(1), dim3(256), 0, st, a, head, slots, gives);
  else hipLaunchKernelGGL((k_plan_scan<16, 4, false>), dim3(1), dim3(1024), 0, st, a, head, slots, gives);
  const int64_t want = (a.max_rows + 1023) / 1024;
  hipLaunchKernelGGL(k_plan_rows, dim3((unsigned)(want < 64 ? 64 : want < 2048 ? want : 2048)), dim3(256), 0, st, a, head, slots, gives);
  return hipGetLastError();
}

}  // namespace awsrc
