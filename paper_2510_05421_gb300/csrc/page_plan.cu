// Page plans: the pages of a paged cache's slots from their lengths.
//
// One cluster does it all, as every slot's pages depend on what the slots before
// it give and take.  Each of its CTAs looks at all slots (a thread a slot) and
// forms the same prefix sums of pages given back, pages taken and rows; then the
// CTAs share the pages that go onto the stack, and behind their barrier those that
// come off it, and the rows.  Nothing is written before the barrier that is read
// after it but the stack, so one barrier is enough.
//
// Bound by its chain: lengths, prefix sums, barrier, stack (2.5 us for 8 slots), then by
// the searches for the rows' slots (64 prompts, 48000 rows: 7 us).
#include "sample.cuh"

namespace dvi {
namespace {

constexpr int kMaxCtas = 8;

struct Shared {
  int back[kPlanSeqs], fresh[kPlanSeqs];   // first of the slot's pages among those given back, taken
  int row[kPlanSeqs + 1];                  // first row
  int len[kPlanSeqs], want[kPlanSeqs], held[kPlanSeqs], need[kPlanSeqs];
  long long part[3][32];
};

// Exclusive prefix sums of three numbers over the CTA's threads, and their totals.
__device__ __forceinline__ void scan3(long long (&v)[3], long long (&total)[3], Shared& s) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
  long long incl[3] = {v[0], v[1], v[2]};
#pragma unroll
  for (int o = 1; o < 32; o <<= 1)
#pragma unroll
    for (int k = 0; k < 3; ++k) {
      const long long w = __shfl_up_sync(0xffffffffu, incl[k], o);
      if (lane >= o) incl[k] += w;
    }
  if (lane == 31)
    for (int k = 0; k < 3; ++k) s.part[k][warp] = incl[k];
  __syncthreads();
  long long sum[3];
#pragma unroll
  for (int k = 0; k < 3; ++k) sum[k] = lane < warps ? s.part[k][lane] : 0;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1)
#pragma unroll
    for (int k = 0; k < 3; ++k) {
      const long long w = __shfl_up_sync(0xffffffffu, sum[k], o);
      if (lane >= o) sum[k] += w;
    }
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    total[k] = __shfl_sync(0xffffffffu, sum[k], 31);
    const long long before = __shfl_sync(0xffffffffu, sum[k], warp ? warp - 1 : 0);
    v[k] = incl[k] - v[k] + (warp ? before : 0);
  }
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

// Slots of blockDim.x threads at most.
__global__ void __launch_bounds__(kPlanSeqs) page_plan_kernel(PagePlanArgs a, int n_ctas) {
  __shared__ Shared s;
  griddep_wait();
  const int b = threadIdx.x, B = a.n_seqs;
  const int rank = blockIdx.x, from = rank * blockDim.x + b, step = n_ctas * blockDim.x;   // this thread's items
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
  long long at[3] = {back, need, rows}, total[3];
  scan3(at, total, s);
  // (more can come back only from a pool that is out of order)
  const int pushed = static_cast<int>(min(total[0], static_cast<long long>(a.n_pages - n_free)));
  if (pushed < total[0]) flags |= DVI_DEV_KV_FULL;
  const int avail = n_free + pushed;
  if (total[1] > avail) {
    // not all can have theirs: slot after slot, what does not fit is passed over
    if (b < B) s.need[b] = need;
    __syncthreads();
    if (b == 0) {
      int left = avail;
      for (int i = 0; i < B; ++i) {
        if (s.need[i] <= left) left -= s.need[i];
        else s.need[i] = -1;
      }
    }
    __syncthreads();
    if (b < B && s.need[b] < 0) {
      flags |= DVI_DEV_KV_FULL;
      need = 0;
    }
    long long again[3] = {0, need, 0}, sums[3];
    scan3(again, sums, s);
    at[1] = again[1];
    total[1] = sums[1];
  }
  const int taken = static_cast<int>(total[1]), all_rows = static_cast<int>(min(total[2], 0x7fffffffll));
  if (b < B) {
    s.back[b] = static_cast<int>(min(at[0], 0x7fffffffll));
    s.fresh[b] = static_cast<int>(at[1]);
    s.row[b] = static_cast<int>(min(at[2], 0x7fffffffll));
    s.len[b] = len;
    s.want[b] = want;
    s.held[b] = held;
    s.need[b] = need;
    if (rank == 0 && a.row_start) a.row_start[b] = s.row[b];
  }
  if (b == 0) {
    s.row[B] = all_rows;
    if (rank == 0 && a.row_start) a.row_start[B] = all_rows;
    if (a.n_rows && total[2] > a.n_rows) flags |= DVI_DEV_KV_FULL;
  }
  __syncthreads();
  for (int i = from; i < pushed; i += step) {
    const int slot = slot_of(s.back, B, i);
    int* entry = a.table + static_cast<int64_t>(slot) * a.max_pages + s.want[slot] + (i - s.back[slot]);
    a.stack[n_free + i] = *entry;
    *entry = -1;
  }
  // the pushed pages are there for all, and all have read what was held
  if (n_ctas > 1) {
    cluster_arrive_release();
    cluster_wait_acquire();
  } else {
    __syncthreads();
  }
  auto page_at = [&](int i) {   // the i-th page taken
    const int page = a.stack[avail - 1 - i];
    return page >= 0 && page < a.n_pages ? page : -1;
  };
  for (int i = from; i < taken; i += step) {
    const int slot = slot_of(s.fresh, B, i);
    const int page = page_at(i);
    if (page < 0) flags |= DVI_DEV_KV_FULL;
    a.table[static_cast<int64_t>(slot) * a.max_pages + s.held[slot] + (i - s.fresh[slot])] = page;
  }
  if (rank == 0) {
    if (b < B) a.held[b] = back ? want : held + need;
    if (b == 0) *a.n_free = avail - taken;
  }
  for (int r = from; r < a.n_rows; r += step) {
    int64_t place = -1;
    int pos = -1;
    if (r < all_rows) {
      const int slot = slot_of(s.row, B, r);
      const int64_t p = static_cast<int64_t>(s.len[slot]) + (r - s.row[slot]), col = p >> a.log_p;
      const int had = s.held[slot];
      int page = -1;
      if (col < had) {
        page = a.table[static_cast<int64_t>(slot) * a.max_pages + col];
      } else if (col < had + s.need[slot]) {
        page = page_at(s.fresh[slot] + static_cast<int>(col) - had);
      }
      if (page >= 0) place = (static_cast<int64_t>(page) << a.log_p) + (p & (P - 1));
      pos = static_cast<int>(min(p, static_cast<int64_t>(0x7fffffff)));
    }
    if (a.slots) a.slots[r] = place;
    if (a.positions) a.positions[r] = pos;
  }
  if (flags) flag_status(a.status, flags);
}

}  // namespace

cudaError_t launch_page_plan(const PagePlanArgs& a, cudaStream_t s) {
  // A CTA's threads: one a slot at least.  More CTAs where there are rows, or slots that may
  // have pages, for them: a plan and a trim of 64 slots with 48000 rows over 8 CTAs 11.1 us, over
  // 4 18.1, over 1 43; of 8 slots with 48 rows over 1 4.9, over 8 5.6.
  const int threads = a.n_seqs <= 256 && a.n_rows <= 2048 ? 256 : kPlanSeqs;
  const int ctas = a.n_rows > 2048 || a.n_seqs > 16 ? kMaxCtas : 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(ctas);
  cfg.blockDim = dim3(threads);
  cfg.stream = s;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = ctas;
  at[1].val.clusterDim.y = 1;
  at[1].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, page_plan_kernel, a, ctas);
}

}  // namespace dvi
