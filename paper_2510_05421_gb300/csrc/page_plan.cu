// Page plans: pages of a paged cache's slots from their lengths, on one CTA.
#include "sample.cuh"

namespace dvi {
namespace {

constexpr int kThreads = kPlanSeqs;   // a slot a thread

struct Shared {
  int back[kPlanSeqs + 1], fresh[kPlanSeqs + 1];   // first of the slot's pages among those given back, taken
  int row[kPlanSeqs + 1];                          // first row
  int len[kPlanSeqs], want[kPlanSeqs], held[kPlanSeqs], need[kPlanSeqs];
  long long part[32];
};

// Exclusive prefix sum over the CTA's threads; *total: the whole.
__device__ long long scan(long long v, Shared& s, long long* total) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  long long incl = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long w = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += w;
  }
  __syncthreads();
  if (lane == 31) s.part[warp] = incl;
  __syncthreads();
  long long base = 0, all = 0;
  for (int w = 0; w < kThreads / 32; ++w) {
    if (w < warp) base += s.part[w];
    all += s.part[w];
  }
  *total = all;
  return base + incl - v;
}

// The last slot whose first item is at most i (first[0] = 0 <= i).
__device__ __forceinline__ int slot_of(const int* first, int n, int i) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (first[mid] <= i) lo = mid;
    else hi = mid;
  }
  return lo;
}

__global__ void __launch_bounds__(kThreads) page_plan_kernel(PagePlanArgs a) {
  __shared__ Shared s;
  griddep_wait();
  const int b = threadIdx.x, B = a.n_seqs;
  const int P = 1 << a.log_p;
  int flags = 0;
  int len = 0, rows = 0, held = 0, want = 0;
  if (b < B) {
    len = max(a.lens[b], 0);
    rows = max(a.rows ? a.rows[b] : a.rows_each, 0);
    const int h = a.held[b];
    held = min(max(h, 0), a.max_pages);
    if (h != held) flags |= DVI_DEV_KV_FULL;
    const long long pages = (static_cast<long long>(len) + rows + P - 1) >> a.log_p;
    want = pages > a.max_pages ? held : static_cast<int>(pages);
    if (pages > a.max_pages) flags |= DVI_DEV_KV_FULL;
  }
  const int n_free = min(max(*a.n_free, 0), a.n_pages);
  const int back = max(held - want, 0);
  int need = max(want - held, 0);
  long long n_back, n_new, n_rows;
  const long long back0 = scan(back, s, &n_back);
  long long new0 = scan(need, s, &n_new);
  const long long row0 = scan(rows, s, &n_rows);
  // (more can come back only from a pool that is out of order)
  const int pushed = static_cast<int>(min(n_back, static_cast<long long>(a.n_pages - n_free)));
  if (pushed < n_back) flags |= DVI_DEV_KV_FULL;
  const int avail = n_free + pushed;
  if (n_new > avail) {
    // not all can have theirs: slot after slot, what does not fit is passed over
    s.need[b] = need;
    __syncthreads();
    if (b == 0) {
      long long left = avail;
      for (int i = 0; i < B; ++i) {
        if (s.need[i] <= left) left -= s.need[i];
        else s.need[i] = -1;
      }
    }
    __syncthreads();
    if (s.need[b] < 0) {
      flags |= DVI_DEV_KV_FULL;
      need = 0;
    }
    new0 = scan(need, s, &n_new);
  }
  if (b < B) {
    s.back[b] = static_cast<int>(min(back0, 0x7fffffffll));
    s.fresh[b] = static_cast<int>(new0);
    s.row[b] = static_cast<int>(min(row0, 0x7fffffffll));
    s.len[b] = len;
    s.want[b] = want;
    s.held[b] = held;
    if (a.row_start) a.row_start[b] = s.row[b];
  }
  if (b == 0) {
    const int all = static_cast<int>(min(n_rows, 0x7fffffffll));
    s.row[B] = all;
    if (a.row_start) a.row_start[B] = all;
    if (a.n_rows && n_rows > a.n_rows) flags |= DVI_DEV_KV_FULL;
    *a.n_free = static_cast<int>(avail - n_new);
  }
  __syncthreads();
  for (int i = b; i < pushed; i += kThreads) {
    const int slot = slot_of(s.back, B, i);
    int* entry = a.table + static_cast<int64_t>(slot) * a.max_pages + s.want[slot] + (i - s.back[slot]);
    a.stack[n_free + i] = *entry;
    *entry = -1;
  }
  __syncthreads();
  for (int i = b; i < n_new; i += kThreads) {
    const int slot = slot_of(s.fresh, B, i);
    const int col = s.held[slot] + (i - s.fresh[slot]);
    int page = a.stack[avail - 1 - i];
    if (page < 0 || page >= a.n_pages) {
      page = -1;
      flags |= DVI_DEV_KV_FULL;
    }
    a.table[static_cast<int64_t>(slot) * a.max_pages + col] = page;
  }
  __syncthreads();   // (the columns above go by what was held)
  if (b < B) a.held[b] = s.held[b] = back ? want : held + need;
  __syncthreads();
  for (int r = b; r < a.n_rows; r += kThreads) {
    int64_t place = -1;
    int pos = -1;
    if (r < s.row[B]) {
      const int slot = slot_of(s.row, B, r);
      const int64_t at = static_cast<int64_t>(s.len[slot]) + (r - s.row[slot]), col = at >> a.log_p;
      if (col < s.held[slot]) {
        const int page = a.table[static_cast<int64_t>(slot) * a.max_pages + col];
        if (page >= 0) place = (static_cast<int64_t>(page) << a.log_p) + (at & (P - 1));
      }
      pos = static_cast<int>(min(at, static_cast<int64_t>(0x7fffffff)));
    }
    if (a.slots) a.slots[r] = place;
    if (a.positions) a.positions[r] = pos;
  }
  if (flags) flag_status(a.status, flags);
}

}  // namespace

cudaError_t launch_page_plan(const PagePlanArgs& a, cudaStream_t s) {
  return launch_pdl(page_plan_kernel, dim3(1), dim3(kThreads), 0, s, a);
}

}  // namespace dvi
