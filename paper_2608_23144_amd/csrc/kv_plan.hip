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
// them.  Small steps run in one launch of one workgroup.
#include "serve_internal.h"

namespace awsrc {

namespace {

// What the scan leaves for the rows: first the header, then one entry per slot.
struct PlanHead {
  int64_t n_free, given, taken, rows;
};
struct PlanSlot {
  int32_t take, give;  // places of its first page among those taken, and among those given back
  int32_t held, want;  // pages before and after
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
  return a.table[s * a.table_ld + plan.slots[s].want + (j - plan.give[s])];
}

// Rows row .. row + 3 of the step, and every step-th four after them.
__device__ __forceinline__ void plan_rows(const PlanArgs& a, const PlanHead& h, const Plan& plan, int64_t first, int64_t step) {
  const int shift = __builtin_ctz(a.pool.page_tokens), P = a.pool.page_tokens;
  for (int64_t row0 = first * 4; row0 < a.max_rows; row0 += step * 4) {
    int32_t seq[4], pos[4];
    int64_t slot[4];
    int s = row0 < h.rows ? last_at_most(a.n_seq, row0, [&](int i) { return plan.cu[i]; }) : 0;
    int32_t start = 0, end = -1, kept = 0, at = -1, page = -1;
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
        start = plan.cu[s];
        end = plan.cu[s + 1];
        kept = a.kv_out[s] - (end - start);
        q = plan.slots[s];
        at = -1;
      }
      seq[i] = s;
      pos[i] = kept + (int32_t)(row - start);
      if (pos[i] >> shift != at) {
        at = pos[i] >> shift;
        int32_t* entry = a.table + s * a.table_ld + at;
        if (at < q.held) {
          page = *entry;
        } else {
          const int64_t t = (int64_t)q.take + at - q.held;
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

// ALONE: the rows too, for at most 64 W slots.
template <int W, bool ALONE>
__global__ __launch_bounds__(64 * W) void k_plan_scan(PlanArgs a, PlanHead* head, PlanSlot* slots, int32_t* gives) {
  __shared__ int64_t sums[3][3][W];
  __shared__ int32_t s_give[ALONE ? 64 * W : 1];
  __shared__ PlanSlot s_slots[ALONE ? 64 * W : 1];
  __shared__ int32_t s_cu[ALONE ? 64 * W + 1 : 1];
  const int shift = __builtin_ctz(a.pool.page_tokens), tid = threadIdx.x;
  int64_t n_free = a.pool.n_free[0];
  n_free = n_free < 0 ? 0 : n_free < a.pool.n_pages ? n_free : a.pool.n_pages;
  const auto read = [&](int s) {
    return s < a.n_seq ? lengths_of(a.kv_len[s], a.keep[s], a.new_len[s], a.table_ld, shift) : Lengths{0, 0, 0, 0};
  };
  // what all slots give back, before anyone is turned away
  Lengths l = read(tid);
  int64_t back[1] = {l.held > l.want ? l.held - l.want : 0}, spare[1];
  for (int s = tid + 64 * W; s < a.n_seq; s += 64 * W) {
    const Lengths m = read(s);
    back[0] += m.held > m.want ? m.held - m.want : 0;
  }
  scan_workgroup<W, 1>(back, spare, sums[0]);
  spare[0] += n_free;
  int64_t asked = 0, queued = 0, rows = 0, taken = 0, given = 0;
  for (int s0 = 0; s0 < a.n_seq; s0 += 64 * W) {
    const int s = s0 + tid;
    if (s0) l = read(s);
    const int64_t need = l.want > l.held ? l.want - l.held : 0;
    int64_t x[2] = {need, l.fresh}, all[2];
    scan_workgroup<W, 2>(x, all, sums[1]);
    const bool served = l.want <= a.table_ld && (need == 0 || asked + x[0] <= spare[0]) && queued + x[1] <= a.max_rows;
    asked += all[0];
    queued += all[1];
    if (!served) {
      l.fresh = 0;
      l.want = pages_of(l.keep, shift);
    }
    const int64_t take = l.want > l.held ? l.want - l.held : 0, give = l.held > l.want ? l.held - l.want : 0;
    int64_t y[3] = {take, give, l.fresh}, sum[3];
    scan_workgroup<W, 3>(y, sum, sums[2]);
    const PlanSlot q = {(int32_t)(taken + y[0] - take), (int32_t)(given + y[1] - give), (int32_t)l.held, (int32_t)l.want};
    if (s < a.n_seq) {
      a.kv_out[s] = (int32_t)(l.keep + l.fresh);
      a.cu[s + 1] = (int32_t)(rows + y[2]);
      if constexpr (ALONE) {
        s_slots[s] = q;
        s_give[s] = q.give;
        s_cu[s + 1] = (int32_t)(rows + y[2]);
      } else {
        slots[s] = q;
        gives[s] = q.give;
      }
    }
    taken += sum[0];
    given += sum[1];
    rows += sum[2];
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
    __threadfence_block();  // (kv_out)
    __syncthreads();
    plan_rows(a, h, Plan{s_slots, s_cu, s_give}, tid, 64 * W);
  }
}

constexpr int kStaged = 2048;  // slots whose starts a workgroup keeps in LDS

__global__ __launch_bounds__(256) void k_plan_rows(PlanArgs a, const PlanHead* head, const PlanSlot* slots, const int32_t* gives) {
  __shared__ int32_t s_cu[kStaged + 1], s_give[kStaged];
  const bool staged = a.n_seq <= kStaged;
  if (staged) {
    for (int i = threadIdx.x; i <= a.n_seq; i += 256) s_cu[i] = a.cu[i];
    for (int i = threadIdx.x; i < a.n_seq; i += 256) s_give[i] = gives[i];
  }
  const PlanHead h = *head;
  __syncthreads();
  const int64_t first = (int64_t)blockIdx.x * 256 + threadIdx.x, step = (int64_t)gridDim.x * 256;
  if (staged) plan_rows(a, h, Plan{slots, s_cu, s_give}, first, step);
  else plan_rows(a, h, Plan{slots, a.cu, gives}, first, step);
}

}  // namespace

size_t kv_plan_ws_bytes(int n_seq) { return n_seq ? 256 + (size_t)n_seq * (sizeof(PlanSlot) + 4) : 0; }

hipError_t launch_kv_plan(const PlanArgs& a, void* ws, hipStream_t st) {
  PlanHead* head = static_cast<PlanHead*>(ws);
  PlanSlot* slots = reinterpret_cast<PlanSlot*>(static_cast<char*>(ws) + 256);
  int32_t* gives = reinterpret_cast<int32_t*>(slots + a.n_seq);
  // One workgroup does it all where its threads have a row or two each.
  if (a.n_seq <= 256 && a.max_rows <= 2048) {
    hipLaunchKernelGGL((k_plan_scan<4, true>), dim3(1), dim3(256), 0, st, a, head, slots, gives);
    return hipGetLastError();
  }
  if (a.n_seq <= 256) hipLaunchKernelGGL((k_plan_scan<4, false>), dim3(1), dim3(256), 0, st, a, head, slots, gives);
  else hipLaunchKernelGGL((k_plan_scan<16, false>), dim3(1), dim3(1024), 0, st, a, head, slots, gives);
  const int64_t want = (a.max_rows + 1023) / 1024;
  hipLaunchKernelGGL(k_plan_rows, dim3((unsigned)(want < 64 ? 64 : want < 2048 ? want : 2048)), dim3(256), 0, st, a, head, slots, gives);
  return hipGetLastError();
}

}  // namespace awsrc
