// Probabilities of sampling from logits: temperature, top-k, top-p.
//
// The CTAs of a cluster hold a row between them (in registers where nothing is cut
// off, else in shared memory), so it is read once.  Without cuts they exchange (max,
// sum of exp2) of every warp once.
//
// With tokens in the order of their logits (equal ones by index) and w =
// exp((x - max) / T), the kept tokens are a prefix of the order; it ends at the
// last token whose rank is below top_k and before which the sum of w is below
// top_p of the whole.  That token is found in two steps: a histogram of counts or
// of w over (max - x) / T gives its bin, and the bin's tokens are sorted out among
// themselves, by every CTA for itself.  Sums of w are whole numbers, so they do not
// depend on the order of the atomics, and every CTA comes to the same end.  Where
// the bin has too many tokens (logits that are nearly equal), the token's place in
// the order, as a number, is found 10 bits at a time over the cluster.
#include <cooperative_groups.h>

#include "sample.cuh"

namespace dvi {
namespace {

namespace cg = cooperative_groups;

constexpr int kThreads = 512;
constexpr int kWarps = kThreads / 32;
constexpr int kMaxCtas = 8;                      // of a row
constexpr int kBins = 1024;
constexpr int kBinBits = 10;
constexpr int kPer = kBins / kThreads;
constexpr float kBinsPerOctave = 40.f;           // of w: the last bin has what is below 2^-25.6
constexpr int kList = 1024;                      // tokens of a bin that are sorted out by each CTA
constexpr int kListPer = kList / kThreads;
constexpr int kFew = 64;                         // tokens that are compared with each other
constexpr int kIndexBits = 18;                   // kMaxVocab

// 2^(k / 32), k = -16 .. 16, as f32 pairs hi + lo.
__constant__ float2 kExp2[33] = {
    {0x1.6a09e6p-1f, 0x1.9fcef4p-27f},  {0x1.71f75ep-1f, 0x1.1d8beep-26f},  {0x1.7a1148p-1f, -0x1.829fd0p-26f},
    {0x1.82589ap-1f, -0x1.accc7cp-27f}, {0x1.8ace54p-1f, 0x1.15506ep-28f},  {0x1.93737cp-1f, -0x1.e64744p-26f},
    {0x1.9c4918p-1f, 0x1.51f848p-28f},  {0x1.a5503cp-1f, -0x1.b83b54p-26f}, {0x1.ae89fap-1f, -0x1.a94b14p-27f},
    {0x1.b7f770p-1f, -0x1.a09438p-26f}, {0x1.c199bep-1f, -0x1.3d56b2p-28f}, {0x1.cb720ep-1f, -0x1.8837ccp-28f},
    {0x1.d5818ep-1f, -0x1.822dbcp-28f}, {0x1.dfc974p-1f, -0x1.908c94p-26f}, {0x1.ea4afap-1f, 0x1.52486cp-28f},
    {0x1.f50766p-1f, -0x1.246eb0p-27f}, {0x1.000000p+0f, 0.f},              {0x1.059b0ep+0f, -0x1.9d4f52p-25f},
    {0x1.0b5586p+0f, 0x1.9f3122p-25f},  {0x1.11301ep+0f, -0x1.fdb496p-25f}, {0x1.172b84p+0f, -0x1.c15742p-27f},
    {0x1.1d4874p+0f, -0x1.d2e8cap-25f}, {0x1.2387a6p+0f, 0x1.ceac48p-25f},  {0x1.29e9e0p+0f, -0x1.5c0424p-25f},
    {0x1.306fe0p+0f, 0x1.4636e2p-25f},  {0x1.371a74p+0f, -0x1.18aac6p-25f}, {0x1.3dea64p+0f, 0x1.824684p-25f},
    {0x1.44e086p+0f, 0x1.8624b4p-30f},  {0x1.4bfdaep+0f, -0x1.593abcp-25f}, {0x1.5342b6p+0f, -0x1.2c5610p-25f},
    {0x1.5ab07ep+0f, -0x1.5bd5ecp-27f}, {0x1.6247ecp+0f, -0x1.f8b550p-25f}, {0x1.6a09e6p+0f, 0x1.9fcef4p-26f}};

// log2(e) / T as an f32 pair, T within 2^-100 .. 2^100.
struct Slope {
  float hi, lo;
};
__device__ __forceinline__ Slope slope_of(float T) {
  const double c = 1.4426950408889634 / static_cast<double>(fminf(fmaxf(T, 0x1p-100f), 0x1p100f));
  const float hi = static_cast<float>(c);
  return {hi, static_cast<float>(c - hi)};
}

// w in f32.
__device__ __forceinline__ float weight(float x, float m, Slope c) { return exp2f((x - m) * c.hi); }

// w in units of 2^-44, off by about 2^-38: x - m and its product with the slope
// as f32 pairs, 2^f by the table and e^z = 1 + z + z^2 (1/2 + z/6 + z^2/24 +
// z^3/120) for |z| <= ln 2 / 64, of which only 1 + z needs the second number.
__device__ __forceinline__ unsigned long long mass(float x, float m, Slope c, const float2* exp2_of) {
  const float dh = __fsub_rn(x, m);
  const float th = __fmul_rn(dh, c.hi);
  if (!(th > -46.f)) return 0;
  const float bb = __fsub_rn(dh, x);
  const float dl = __fadd_rn(__fsub_rn(x, __fsub_rn(dh, bb)), __fsub_rn(-m, bb));
  const float tl = fmaf(dh, c.hi, -th) + fmaf(dh, c.lo, dl * c.hi);
  const float n = rintf(th);
  const float f = __fsub_rn(th, n);
  const float k = rintf(f * 32.f);
  const float r = fmaf(k, -0.03125f, f);
  const float kLn2 = 0x1.62e430p-1f, kLn2Lo = -0x1.05c610p-29f;
  const float z = __fmul_rn(r, kLn2);
  const float zl = fmaf(r, kLn2, -z) + fmaf(r, kLn2Lo, tl * kLn2);
  const float q = z * z * fmaf(z, fmaf(z, fmaf(z, 1.f / 120.f, 1.f / 24.f), 1.f / 6.f), 0.5f);
  const float p = __fadd_rn(z, q);
  const float pl = __fadd_rn(__fsub_rn(z, p), q) + fmaf(z, zl, zl);
  const float2 t = exp2_of[static_cast<int>(k) + 16];
  const float prod = __fmul_rn(t.x, p);
  const float e = fmaf(t.x, p, -prod) + fmaf(t.x, pl, t.y);
  const float hi = __fadd_rn(t.x, prod);
  const float lo = __fadd_rn(__fsub_rn(t.x, hi), prod) + e;
  // 22 bits, then 22 more of what they leave
  const float s = __int_as_float((static_cast<int>(n) + 22 + 127) << 23);
  const float h = hi * s;
  const float a = floorf(h);
  const float b = rintf(fmaf(lo, s, __fsub_rn(h, a)) * 4194304.f);
  return (static_cast<unsigned long long>(static_cast<unsigned>(a)) << 22) + static_cast<long long>(static_cast<int>(b));
}

// f32 as a number that grows with it, and back.
__device__ __forceinline__ uint32_t ord(float x) {
  const uint32_t b = __float_as_uint(x);
  return (b & 0x80000000u) ? ~b : (b | 0x80000000u);
}
__device__ __forceinline__ float from_ord(uint32_t o) {
  return __uint_as_float((o & 0x80000000u) ? (o & 0x7fffffffu) : ~o);
}

// A logit as it counts: NaN as -inf, +inf as the largest number, -0 as 0.
__device__ __forceinline__ float clean(float v) { return v != v ? -INFINITY : fminf(v, 3.402823466e38f) + 0.f; }

__device__ __forceinline__ unsigned long long warp_sum_u64(unsigned long long v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// What a row with cuts needs beside its slice of logits.
struct Cuts {
  unsigned lo[kBins], hi[kBins];            // sums of the bins
  unsigned long long list[kList];           // this CTA's tokens of the chosen bin
  unsigned long long key[kList], mass[kList];   // the cluster's
};

struct Small {
  float2 exp2_of[33];
  Slope slope;
  unsigned long long part[kWarps], least[kWarps], most[kWarps];
  // written by the warps of the cluster: (max, sum), or (max, first token of it)
  float2 peer[kMaxCtas * kWarps];
  unsigned long long peer_sum[2][kMaxCtas];
  int n_list[2], n_kept;
  int found;
  unsigned long long excl, cut, kept;
};

// One row (its slice in this CTA) and what is known of it.
struct RowState {
  const float* x;       // the slice, tokens first .. first + n - 1
  int first, n;
  float m;              // the row's maximum
  uint32_t top;         // ord(m)
  Slope c;
  __device__ __forceinline__ unsigned long long place(float v, int i) const {
    return (static_cast<unsigned long long>(top - ord(v)) << kIndexBits) | static_cast<unsigned>(first + i);
  }
  __device__ __forceinline__ float logit(unsigned long long place) const {
    return from_ord(top - static_cast<uint32_t>(place >> kIndexBits));
  }
  __device__ __forceinline__ int bin(float v) const {
    const float t = __fmul_rn(__fmul_rn(__fsub_rn(m, v), c.hi), kBinsPerOctave);
    return static_cast<int>(fminf(t, static_cast<float>(kBins - 1)));
  }
};

__device__ __forceinline__ void cluster_barrier(int n_ctas) {
  if (n_ctas > 1) {
    cluster_arrive_release();
    cluster_wait_acquire();
  } else {
    __syncthreads();
  }
}

// Gives the sum over this CTA to all of the cluster: peer_sum[slot] is complete behind
// the next cluster_barrier.  `slot` is of its own for each call.
__device__ __forceinline__ void give_sum(unsigned long long v, int slot, int rank, int n_ctas, Small& s) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  v = warp_sum_u64(v);
  if (lane == 0) s.part[warp] = v;
  __syncthreads();
  if (warp == 0) {
    v = warp_sum_u64(lane < kWarps ? s.part[lane] : 0);
    if (lane < n_ctas) *cg::this_cluster().map_shared_rank(&s.peer_sum[slot][rank], lane) = v;
  }
}
__device__ __forceinline__ unsigned long long given_sum(int slot, int n_ctas, const Small& s) {
  unsigned long long v = 0;
  for (int r = 0; r < n_ctas; ++r) v += s.peer_sum[slot][r];
  return v;
}

// Adds to a bin's 64-bit sum; the 32-bit halves are exact together whatever the order.
__device__ __forceinline__ void add_to_bin(Cuts& h, int bin, unsigned long long v) {
  const unsigned lo = static_cast<unsigned>(v), old = atomicAdd(&h.lo[bin], lo);
  const unsigned up = static_cast<unsigned>(v >> 32) + (old + lo < old ? 1u : 0u);
  if (up) atomicAdd(&h.hi[bin], up);
}

__device__ __forceinline__ void clear_bins(Cuts& h) {
  for (int i = threadIdx.x; i < kBins; i += kThreads) h.lo[i] = 0, h.hi[i] = 0;
  __syncthreads();
}

// The first bin up to which the sums of CTAs r0 .. r1 - 1 (and `before`) reach target: its
// number (-1 if none does) and the sum before it.  Their bins are complete when it is called.
__device__ int find_bin(unsigned long long before, unsigned long long target, int r0, int r1, Cuts& h, Small& s,
                        unsigned long long* excl) {
  cg::cluster_group cluster = cg::this_cluster();
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  unsigned long long v[kPer] = {}, sum = 0;
  static_assert(kPer == 2, "a pair of bins a thread");
  for (int r = r0; r < r1; ++r) {
    const uint2 lo = reinterpret_cast<const uint2*>(cluster.map_shared_rank(h.lo, r))[tid];
    const uint2 hi = reinterpret_cast<const uint2*>(cluster.map_shared_rank(h.hi, r))[tid];
    v[0] += (static_cast<unsigned long long>(hi.x) << 32) + lo.x;
    v[1] += (static_cast<unsigned long long>(hi.y) << 32) + lo.y;
  }
#pragma unroll
  for (int j = 0; j < kPer; ++j) sum += v[j];
  unsigned long long incl = sum;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const unsigned long long w = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += w;
  }
  if (lane == 31) s.part[warp] = incl;
  if (tid == 0) s.found = -1;
  __syncthreads();
  unsigned long long at = before + incl - sum;
  for (int w = 0; w < warp; ++w) at += s.part[w];
#pragma unroll
  for (int j = 0; j < kPer; ++j) {
    if (at < target && at + v[j] >= target) s.found = tid * kPer + j, s.excl = at;
    at += v[j];
  }
  __syncthreads();
  *excl = s.excl;
  return s.found;
}

// Of the n tokens in h.key (with h.mass): the last kept one, where `before` is the sum before
// them all.  By every CTA for itself.
template <bool MASS>
__device__ unsigned long long last_of_list(int n, unsigned long long before, unsigned long long target, int rank,
                                           Cuts& h, Small& s, unsigned long long* kept) {
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  while (n > kFew) {
    // bins of equal width from the first of their places to the last
    unsigned long long key[kListPer], m[kListPer], least = ~0ull, most = 0;
#pragma unroll
    for (int j = 0; j < kListPer; ++j) {
      const int i = tid + j * kThreads;
      key[j] = i < n ? h.key[i] : ~0ull;
      m[j] = i < n && MASS ? h.mass[i] : 1;
      if (i < n) least = min(least, key[j]), most = max(most, key[j]);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      least = min(least, __shfl_xor_sync(0xffffffffu, least, o));
      most = max(most, __shfl_xor_sync(0xffffffffu, most, o));
    }
    if (lane == 0) s.least[warp] = least, s.most[warp] = most;
    if (tid == 0) s.n_kept = 0;
    clear_bins(h);
    for (int w = 0; w < kWarps; ++w) least = min(least, s.least[w]), most = max(most, s.most[w]);
    const int bits = 64 - __clzll(most - least), shift = bits > kBinBits ? bits - kBinBits : 0;
#pragma unroll
    for (int j = 0; j < kListPer; ++j)
      if (key[j] != ~0ull) add_to_bin(h, static_cast<int>((key[j] - least) >> shift), m[j]);
    __syncthreads();
    const int bin = find_bin(before, target, rank, rank + 1, h, s, &before);
#pragma unroll
    for (int j = 0; j < kListPer; ++j) {
      if (key[j] == ~0ull || static_cast<int>((key[j] - least) >> shift) != bin) continue;
      const int at = atomicAdd(&s.n_kept, 1);
      h.key[at] = key[j];
      if (MASS) h.mass[at] = m[j];
    }
    __syncthreads();
    n = s.n_kept;
    __syncthreads();
  }
  if (tid < n) {
    const unsigned long long p = h.key[tid], v = MASS ? h.mass[tid] : 1;
    unsigned long long sum = before;
    for (int j = 0; j < n; ++j)
      if (h.key[j] < p) sum += MASS ? h.mass[j] : 1;
    if (sum < target && sum + v >= target) s.cut = p, s.kept = sum + v;
  }
  __syncthreads();
  *kept = s.kept;
  return s.cut;
}

// ceil(p S) for p in [0, 1), at least 1.
__device__ __forceinline__ unsigned long long share_of(float p, unsigned long long S) {
  const uint32_t b = __float_as_uint(p);
  const int e = static_cast<int>(b >> 23);
  const unsigned long long f = e ? (b & 0x7fffffu) | 0x800000u : b & 0x7fffffu;
  const int shift = 150 - (e ? e : 1);                   // p = f 2^-shift, shift >= 24
  const unsigned long long lo = S * f, hi = __umul64hi(S, f);
  unsigned long long t;
  if (shift < 64)
    t = (hi << (64 - shift)) + (lo >> shift) + ((lo & ((1ull << shift) - 1)) ? 1 : 0);
  else
    t = shift < 128 ? (hi >> (shift - 64)) + 1 : 1;      // (one too many where nothing is left over: below 2^-40 of S)
  return t ? t : 1;
}

// The place of the last kept token among those up to the place `upto`: before it the counts
// sum to less than top_k, or (MASS) the masses to less than top_p of all.  *kept: the sum up
// to it (that of all where it is ~0: all are kept).  Tokens below `least` are known to be cut.
// mine: the largest of the thread's own logits.
template <bool MASS>
__device__ unsigned long long last_kept(const RowState& row, int top_k, float top_p, unsigned long long upto,
                                        float least, float mine, int rank, int n_ctas, Cuts& h, Small& s,
                                        unsigned long long* kept) {
  cg::cluster_group cluster = cg::this_cluster();
  const int tid = threadIdx.x;
  unsigned long long before;
  clear_bins(h);
  int most = kBins - 1;
  if (!MASS && top_k <= kThreads) {
    // top_k threads' largest logits are in the first bins: no token behind these is kept
    if (mine > -INFINITY) atomicAdd(&h.lo[row.bin(mine)], 1u);
    __syncthreads();
    const int b = find_bin(0, top_k, rank, rank + 1, h, s, &before);
    if (b >= 0) most = b;
    clear_bins(h);
  }
  auto counts = [&](float x, int i) { return x > -INFINITY && x >= least && (upto == ~0ull || row.place(x, i) <= upto); };
  if (MASS) {
    unsigned long long all = 0;
    for (int i = tid; i < row.n; i += kThreads) {
      const float x = row.x[i];
      if (upto != ~0ull && row.place(x, i) > upto) continue;
      const unsigned long long m = mass(x, row.m, row.c, s.exp2_of);
      all += m;
      if (x >= least && m) add_to_bin(h, row.bin(x), m);
    }
    give_sum(all, 1, rank, n_ctas, s);
  } else {
    for (int i = tid; i < row.n; i += kThreads) {
      const float x = row.x[i];
      if (!(x > -INFINITY)) continue;
      const int bin = row.bin(x);
      if (bin <= most) atomicAdd(&h.lo[bin], 1u);
    }
  }
  cluster_barrier(n_ctas);
  unsigned long long target = top_k;
  if (MASS) {
    *kept = given_sum(1, n_ctas, s);
    target = share_of(top_p, *kept);
  }
  const int bin = find_bin(0, target, 0, n_ctas, h, s, &before);
  if (bin < 0) return ~0ull;
  int& found = s.n_list[MASS];
  for (int i = tid; i < row.n; i += kThreads) {
    const float x = row.x[i];
    if (row.bin(x) != bin || !counts(x, i)) continue;
    const int at = atomicAdd(&found, 1);
    if (at < kList) h.list[at] = row.place(x, i);
  }
  cluster_barrier(n_ctas);
  int n = 0;
  for (int r = 0; r < n_ctas; ++r) n += *cluster.map_shared_rank(&found, r);
  if (n <= kList) {
    for (int r = 0, at = 0; r < n_ctas; ++r) {
      const int there = *cluster.map_shared_rank(&found, r);
      const unsigned long long* list = cluster.map_shared_rank(h.list, r);
      for (int i = tid; i < there; i += kThreads) {
        const unsigned long long p = list[i];
        h.key[at + i] = p;
        if (MASS) h.mass[at + i] = mass(row.logit(p), row.m, row.c, s.exp2_of);
      }
      at += there;
    }
    __syncthreads();
    return last_of_list<MASS>(n, before, target, rank, h, s, kept);
  }
  unsigned long long lo = 0;
  before = 0;
  for (int shift = 32 + kIndexBits - kBinBits;; shift = shift > kBinBits ? shift - kBinBits : 0) {
    clear_bins(h);
    for (int i = tid; i < row.n; i += kThreads) {
      const float x = row.x[i];
      if (!counts(x, i)) continue;
      const unsigned long long p = row.place(x, i);
      if (p < lo || ((p - lo) >> shift) >= kBins) continue;
      add_to_bin(h, static_cast<int>((p - lo) >> shift), MASS ? mass(x, row.m, row.c, s.exp2_of) : 1ull);
    }
    cluster_barrier(n_ctas);
    const int b = find_bin(before, target, 0, n_ctas, h, s, &before);   // (found: the sums are those of the first bins)
    lo += static_cast<unsigned long long>(b) << shift;
    if (shift == 0) {
      // one token a bin
      unsigned long long v = 0;
      for (int r = 0; r < n_ctas; ++r)
        v += (static_cast<unsigned long long>(cluster.map_shared_rank(h.hi, r)[b]) << 32) +
             cluster.map_shared_rank(h.lo, r)[b];
      *kept = before + v;
      cluster_barrier(n_ctas);
      return lo;
    }
    cluster_barrier(n_ctas);   // before the bins are cleared
  }
}

// The settings of row r, as they count.
struct Settings {
  float temperature, top_p;   // 0: greedy; 1: no cut
  int top_k;                  // 0: no cut
  bool bad;
  __device__ __forceinline__ Settings(const TokenProbsArgs& a, int r) {
    temperature = a.temperature ? a.temperature[r] : a.temperature_all;
    top_p = a.top_p ? a.top_p[r] : a.top_p_all;
    top_k = a.top_k ? a.top_k[r] : a.top_k_all;
    bad = temperature != temperature || top_p != top_p;
    if (!(temperature > 0.f)) temperature = 0.f;
    top_p = top_p < 1.f ? fmaxf(top_p, 0.f) : 1.f;
    if (top_k < 0 || top_k >= a.vocab) top_k = 0;
  }
};

// What all warps of the cluster have given: the row's maximum and its sum of w (T > 0) or its
// first largest token (T = 0).
__device__ __forceinline__ void join(const Small& s, int n_ctas, bool greedy, Slope c, float* m, float* sum, int* hot) {
  const int lane = threadIdx.x & 31;
  float top = -INFINITY;
  for (int i = lane; i < n_ctas * kWarps; i += 32) top = fmaxf(top, s.peer[i].x);
  top = warp_max(top);
  float all = 0.f;
  int first = 0x7fffffff;
  for (int i = lane; i < n_ctas * kWarps; i += 32) {
    const float2 p = s.peer[i];
    if (greedy) {
      if (p.x == top) first = min(first, __float_as_int(p.y));
    } else if (p.x > -INFINITY) {
      all += p.y * weight(p.x, top, c);
    }
  }
  *m = top;
  *sum = warp_sum(all);
  *hot = __reduce_min_sync(0xffffffffu, first);
}

// Rows without cuts: NV logits a thread, in registers.
template <typename T, int NV>
__global__ void __launch_bounds__(kThreads, NV <= 16 ? 3 : NV <= 32 ? 2 : 1)
    token_probs_kernel(TokenProbsArgs a, int n_ctas, int slice) {
  __shared__ Small s;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int rank = n_ctas > 1 ? static_cast<int>(cg::this_cluster().block_rank()) : 0;
  const int r = blockIdx.x / n_ctas;
  const int first = min(rank * slice, a.vocab), n = min(slice, a.vocab - first);
  if (n_ctas > 1) cluster_arrive_release();              // (waited for below: no CTA writes to one that is not there)
  griddep_wait();
  const T* in = static_cast<const T*>(a.x) + r * a.ld + first;
  float* out = a.out + r * a.ld_out + first;
  float v[NV];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int i = j * kThreads + tid;
    v[j] = i < n ? DT<T>::ld(in + i) : -INFINITY;
  }
  const Settings set(a, r);
  const bool greedy = set.temperature == 0.f;
  if (tid == 0) s.slope = slope_of(set.temperature);
  bool bad = set.bad;
  float m = -INFINITY;
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    bad |= !(v[j] < INFINITY);
    v[j] = clean(v[j]);
    m = fmaxf(m, v[j]);
  }
  m = warp_max(m);
  if (__syncthreads_or(bad) && tid == 0) flag_status(a.status, DVI_DEV_NONFINITE);
  const Slope c = s.slope;
  float2 mine = make_float2(m, 0.f);
  if (greedy) {
    int at = 0x7fffffff;
#pragma unroll
    for (int j = NV - 1; j >= 0; --j)
      if (v[j] == m) at = first + j * kThreads + tid;
    mine.y = __int_as_float(__reduce_min_sync(0xffffffffu, at));
  } else if (m > -INFINITY) {
    float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < NV; ++j) sum[j & 3] += v[j] = weight(v[j], m, c);
    mine.y = warp_sum((sum[0] + sum[1]) + (sum[2] + sum[3]));
  }
  if (n_ctas > 1) {
    cluster_wait_acquire();
    if (lane < n_ctas) *cg::this_cluster().map_shared_rank(&s.peer[rank * kWarps + warp], lane) = mine;
  } else if (lane == 0) {
    s.peer[warp] = mine;
  }
  cluster_barrier(n_ctas);
  float top, sum;
  int hot;
  join(s, n_ctas, greedy, c, &top, &sum, &hot);
  const float scale = !greedy && m > -INFINITY ? weight(m, top, c) / sum : 0.f;
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int i = j * kThreads + tid;
    if (i < n) out[i] = scale > 0.f ? v[j] * scale : greedy && top > -INFINITY && first + i == hot ? 1.f : 0.f;
  }
}

// Rows with cuts: a slice in shared memory.
template <typename T>
__global__ void __launch_bounds__(kThreads, 2) token_probs_cut_kernel(TokenProbsArgs a, int n_ctas, int slice) {
  extern __shared__ __align__(16) unsigned char dynamic[];
  __shared__ Small s;
  Cuts& h = *reinterpret_cast<Cuts*>(dynamic);
  float* x = reinterpret_cast<float*>(dynamic + sizeof(Cuts));
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int rank = n_ctas > 1 ? static_cast<int>(cg::this_cluster().block_rank()) : 0;
  const int r = blockIdx.x / n_ctas;
  const int first = min(rank * slice, a.vocab), n = min(slice, a.vocab - first);
  if (n_ctas > 1) cluster_arrive_release();
  griddep_wait();
  const T* in = static_cast<const T*>(a.x) + r * a.ld + first;
  float* out = a.out + r * a.ld_out + first;
  const Settings set(a, r);
  const bool greedy = set.temperature == 0.f;
  bool bad = set.bad;
  if (tid == 0) {
    s.slope = slope_of(set.temperature);
    s.n_list[0] = s.n_list[1] = 0;
  }
  if (tid >= 64 && tid < 64 + 33) s.exp2_of[tid - 64] = kExp2[tid - 64];

  constexpr int kFly = 16;
  float own = -INFINITY;
  int at = 0x7fffffff;
  for (int i0 = 0; i0 < n; i0 += kFly * kThreads) {
    float v[kFly];
#pragma unroll
    for (int j = 0; j < kFly; ++j) {
      const int i = i0 + j * kThreads + tid;
      v[j] = i < n ? DT<T>::ld(in + i) : -INFINITY;
    }
#pragma unroll
    for (int j = 0; j < kFly; ++j) {
      const int i = i0 + j * kThreads + tid;
      bad |= !(v[j] < INFINITY);
      v[j] = clean(v[j]);
      if (v[j] > own) own = v[j], at = first + i;
      if (i < n) x[i] = v[j];
    }
  }
  const float m = warp_max(own);
  if (__syncthreads_or(bad) && tid == 0) flag_status(a.status, DVI_DEV_NONFINITE);
  const Slope c = s.slope;
  // (of the sum of w the largest logits of the threads: a lower bound is enough)
  float2 mine = make_float2(m, 0.f);
  if (greedy)
    mine.y = __int_as_float(__reduce_min_sync(0xffffffffu, own == m ? at : 0x7fffffff));
  else if (m > -INFINITY)
    mine.y = warp_sum(weight(own, m, c));
  if (n_ctas > 1) {
    cluster_wait_acquire();
    if (lane < n_ctas) *cg::this_cluster().map_shared_rank(&s.peer[rank * kWarps + warp], lane) = mine;
  } else if (lane == 0) {
    s.peer[warp] = mine;
  }
  cluster_barrier(n_ctas);
  float top, sum;
  int hot;
  join(s, n_ctas, greedy, c, &top, &sum, &hot);
  if (greedy || top == -INFINITY) {
    for (int i = tid; i < n; i += kThreads) out[i] = top > -INFINITY && first + i == hot ? 1.f : 0.f;
    return;
  }
  const RowState row = {x, first, n, top, ord(top), c};
  unsigned long long upto = ~0ull, kept = 0;
  if (set.top_k)
    upto = last_kept<false>(row, set.top_k, 1.f, ~0ull, -INFINITY, own, rank, n_ctas, h, s, &kept);
  if (set.top_p < 1.f) {
    // tokens below (1 - p) S / V sum to less than what may be cut, so the last kept one is
    // above that (half of it, for the sum's rounding)
    float least = -INFINITY;
    if (upto == ~0ull)
      least = top + log2f(0.5f * (1.f - set.top_p) * sum / static_cast<float>(a.vocab)) / c.hi * 1.0001f;
    const unsigned long long e = last_kept<true>(row, 0, set.top_p, upto, least, own, rank, n_ctas, h, s, &kept);
    if (e != ~0ull) upto = e;
  } else {
    unsigned long long all = 0;
    for (int i = tid; i < n; i += kThreads)
      if (upto == ~0ull || row.place(x[i], i) <= upto) all += mass(x[i], top, c, s.exp2_of);
    give_sum(all, 0, rank, n_ctas, s);
    cluster_barrier(n_ctas);
    kept = given_sum(0, n_ctas, s);
  }
  if (n_ctas > 1) cluster_arrive_release();   // nothing of the others is read from here on
  const float inv = 1.f / (__ull2float_rn(kept) * 0x1p-44f);
  const float x_cut = upto == ~0ull ? -INFINITY : row.logit(upto);
  const int i_cut = static_cast<int>(upto & ((1u << kIndexBits) - 1)) - first;
  for (int i = tid; i < n; i += kThreads) {
    const float v = x[i];
    const bool in_it = v > x_cut || (v == x_cut && i <= i_cut && v > -INFINITY);
    out[i] = in_it ? weight(v, top, c) * inv : 0.f;
  }
  if (n_ctas > 1) cluster_wait_acquire();     // (and no CTA leaves while another may read what it found)
}

template <typename K>
cudaError_t launch(K kern, const TokenProbsArgs& a, int ctas, size_t smem, cudaStream_t s) {
  if (static_cast<int64_t>(a.n_rows) * ctas > 0x7fffffffll) return cudaErrorInvalidConfiguration;
  const int slice = (a.vocab + ctas - 1) / ctas;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(a.n_rows) * ctas);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = smem ? smem + slice * sizeof(float) : 0;
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
  return cudaLaunchKernelEx(&cfg, kern, a, ctas, slice);
}

template <typename T>
cudaError_t launch_plain(const TokenProbsArgs& a, cudaStream_t s) {
  int nv = 16;
  while (nv * kThreads * kMaxCtas < a.vocab) nv *= 2;
  int ctas = 1;
  while (ctas * nv * kThreads < a.vocab) ctas *= 2;
  if (nv == 16) return launch(token_probs_kernel<T, 16>, a, ctas, 0, s);
  return nv == 32 ? launch(token_probs_kernel<T, 32>, a, ctas, 0, s) : launch(token_probs_kernel<T, 64>, a, ctas, 0, s);
}

constexpr int kSlice = 16384;   // logits of a CTA where its row may have up to kMaxCtas: two CTAs an SM

template <typename T>
cudaError_t launch_cut(const TokenProbsArgs& a, cudaStream_t s) {
  static PerDevice per_device;
  per_device.once([&] {
    cudaFuncSetAttribute(token_probs_cut_kernel<T>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                         kMaxVocab / kMaxCtas * static_cast<int>(sizeof(float)) + static_cast<int>(sizeof(Cuts)));
  });
  int ctas = 1;
  while (ctas < kMaxCtas && (ctas * kSlice < a.vocab || (static_cast<int64_t>(a.n_rows) * ctas < 152 && a.vocab / ctas > 4096)))
    ctas *= 2;
  return launch(token_probs_cut_kernel<T>, a, ctas, sizeof(Cuts), s);
}

}  // namespace

cudaError_t launch_token_probs(const TokenProbsArgs& a, int dtype, cudaStream_t s) {
  const bool cuts = a.top_k || a.top_p || a.top_p_all < 1.f || (a.top_k_all > 0 && a.top_k_all < a.vocab);
  if (dtype == DVI_BF16) return cuts ? launch_cut<__nv_bfloat16>(a, s) : launch_plain<__nv_bfloat16>(a, s);
  return cuts ? launch_cut<float>(a, s) : launch_plain<float>(a, s);
}

}  // namespace dvi
