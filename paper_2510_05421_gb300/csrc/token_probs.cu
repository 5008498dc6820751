// Probabilities of sampling from logits: temperature, top-k, top-p.
//
// A row's slices lie in the shared memory of one cluster's CTAs, so the row is
// read once; the CTAs exchange (max, sum of exp2) once, which is all that a row
// without cuts needs.
//
// With tokens in the order of their logits (equal ones by index) and w =
// exp((x - max) / T), the kept tokens are a prefix of the order; it ends at the
// last token whose rank is below top_k and before which the sum of w is below
// top_p of the whole.  That token is found in two steps: a histogram of counts or
// of w over (max - x) / T gives its bin, and the bin's tokens are compared with
// each other.  Sums of w are whole numbers, so they do not depend on the order of
// the atomics, and every CTA of the cluster comes to the same end.  Where the bin
// has too many tokens (logits that are nearly equal), the token's place in the
// order, as a number, is found 11 bits at a time.
#include <cooperative_groups.h>

#include "sample.cuh"

namespace dvi {
namespace {

namespace cg = cooperative_groups;

constexpr int kThreads = 512;
constexpr int kWarps = kThreads / 32;
constexpr int kMaxCtas = 8;                      // of a row
constexpr int kBins = 2048;
constexpr int kBinBits = 11;
constexpr int kPer = kBins / kThreads;
constexpr float kBinsPerOctave = 64.f;           // of w: the last bin has what is below 2^-32
constexpr int kList = 1024;                      // tokens of a bin that are compared with each other
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
  float red[kWarps], sum[kWarps];
  int first[kWarps];
  unsigned long long part[kWarps];
  // written by the CTAs of the cluster, by rank
  float2 peer[kMaxCtas];                    // (max, sum)
  int peer_first[kMaxCtas];
  unsigned long long peer_sum[2][kMaxCtas];
  int n_list[2];
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

// Sum over the cluster; `slot` is of its own for each call.
__device__ unsigned long long cluster_sum(unsigned long long v, int slot, int n_ctas, Small& s) {
  cg::cluster_group cluster = cg::this_cluster();
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  v = warp_sum_u64(v);
  if (lane == 0) s.part[warp] = v;
  __syncthreads();
  if (warp == 0) {
    v = warp_sum_u64(lane < kWarps ? s.part[lane] : 0);
    if (lane < n_ctas) *cluster.map_shared_rank(&s.peer_sum[slot][cluster.block_rank()], lane) = v;
  }
  cluster_barrier(n_ctas);
  v = 0;
  for (int r = 0; r < n_ctas; ++r) v += s.peer_sum[slot][r];
  return v;
}

// Adds to a bin's 64-bit sum; the 32-bit halves are exact together whatever the order.
__device__ __forceinline__ void add_to_bin(Cuts& h, int bin, unsigned long long v) {
  const unsigned lo = static_cast<unsigned>(v), old = atomicAdd(&h.lo[bin], lo);
  const unsigned up = static_cast<unsigned>(v >> 32) + (old + lo < old ? 1u : 0u);
  if (up) atomicAdd(&h.hi[bin], up);
}

// The first bin up to which the cluster's sums (and `before`) reach target: its number
// (-1 if none does) and the sum before it.  Every CTA's bins are complete when it is called.
__device__ int find_bin(unsigned long long before, unsigned long long target, int n_ctas, Cuts& h, Small& s,
                        unsigned long long* excl) {
  cg::cluster_group cluster = cg::this_cluster();
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  unsigned long long v[kPer] = {}, sum = 0;
  for (int r = 0; r < n_ctas; ++r) {
    const uint4 lo = reinterpret_cast<const uint4*>(cluster.map_shared_rank(h.lo, r))[tid];
    const uint4 hi = reinterpret_cast<const uint4*>(cluster.map_shared_rank(h.hi, r))[tid];
    v[0] += (static_cast<unsigned long long>(hi.x) << 32) + lo.x;
    v[1] += (static_cast<unsigned long long>(hi.y) << 32) + lo.y;
    v[2] += (static_cast<unsigned long long>(hi.z) << 32) + lo.z;
    v[3] += (static_cast<unsigned long long>(hi.w) << 32) + lo.w;
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

// The place of the last kept token: before it the counts (MASS: the masses), over tokens
// up to the place `upto`, sum to less than target.  *kept: the sum up to it.  ~0 if the
// whole sum is less than target.  MASS: tokens below `least` are known to be cut.
template <bool MASS>
__device__ unsigned long long last_kept(const RowState& row, unsigned long long target, unsigned long long upto,
                                        float least, int n_ctas, Cuts& h, Small& s, unsigned long long* kept) {
  cg::cluster_group cluster = cg::this_cluster();
  const int tid = threadIdx.x;
  auto zero = [&] {
    for (int i = tid; i < kBins; i += kThreads) h.lo[i] = 0, h.hi[i] = 0;
    __syncthreads();
  };
  auto counts = [&](float x, int i) {
    if (x == -INFINITY || (MASS && weight(x, row.m, row.c) < least)) return false;
    return upto == ~0ull || row.place(x, i) <= upto;
  };
  zero();
  for (int i = tid; i < row.n; i += kThreads) {
    const float x = row.x[i];
    if (!counts(x, i)) continue;
    if (MASS)
      add_to_bin(h, row.bin(x), mass(x, row.m, row.c, s.exp2_of));
    else
      atomicAdd(&h.lo[row.bin(x)], 1u);
  }
  cluster_barrier(n_ctas);
  unsigned long long before;
  const int bin = find_bin(0, target, n_ctas, h, s, &before);
  if (bin < 0) return ~0ull;
  int& mine = s.n_list[MASS];
  for (int i = tid; i < row.n; i += kThreads) {
    const float x = row.x[i];
    if (!counts(x, i) || row.bin(x) != bin) continue;
    const int at = atomicAdd(&mine, 1);
    if (at < kList) h.list[at] = row.place(x, i);
  }
  cluster_barrier(n_ctas);
  int n = 0;
  for (int r = 0; r < n_ctas; ++r) n += *cluster.map_shared_rank(&mine, r);
  if (n <= kList) {
    for (int r = 0, at = 0; r < n_ctas; ++r) {
      const int there = *cluster.map_shared_rank(&mine, r);
      const unsigned long long* list = cluster.map_shared_rank(h.list, r);
      for (int i = tid; i < there; i += kThreads) {
        const unsigned long long p = list[i];
        h.key[at + i] = p;
        if (MASS) h.mass[at + i] = mass(from_ord(row.top - static_cast<uint32_t>(p >> kIndexBits)), row.m, row.c, s.exp2_of);
      }
      at += there;
    }
    __syncthreads();
    for (int i = tid; i < n; i += kThreads) {
      const unsigned long long p = h.key[i], v = MASS ? h.mass[i] : 1;
      unsigned long long sum = before;
      for (int j = 0; j < n; ++j)
        if (h.key[j] < p) sum += MASS ? h.mass[j] : 1;
      if (sum < target && sum + v >= target) s.cut = p, s.kept = sum + v;
    }
    __syncthreads();
    *kept = s.kept;
    return s.cut;
  }
  unsigned long long lo = 0;
  before = 0;
  for (int shift = 32 + kIndexBits - kBinBits;; shift = shift > kBinBits ? shift - kBinBits : 0) {
    zero();
    for (int i = tid; i < row.n; i += kThreads) {
      const float x = row.x[i];
      if (!counts(x, i)) continue;
      const unsigned long long p = row.place(x, i);
      if (p < lo || ((p - lo) >> shift) >= kBins) continue;
      add_to_bin(h, static_cast<int>((p - lo) >> shift), MASS ? mass(x, row.m, row.c, s.exp2_of) : 1ull);
    }
    cluster_barrier(n_ctas);
    unsigned long long excl;
    const int b = find_bin(before, target, n_ctas, h, s, &excl);   // (found: the sums are those of the first bins)
    lo += static_cast<unsigned long long>(b) << shift;
    before = excl;
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

template <typename T, bool CUTS>
__global__ void __launch_bounds__(kThreads, 2) token_probs_kernel(TokenProbsArgs a, int n_ctas, int slice) {
  extern __shared__ __align__(16) unsigned char dynamic[];
  __shared__ Small s;
  float* x = reinterpret_cast<float*>(dynamic);
  Cuts& h = *reinterpret_cast<Cuts*>(dynamic + (static_cast<size_t>(slice) * sizeof(float) + 15) / 16 * 16);
  cg::cluster_group cluster = cg::this_cluster();
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int rank = n_ctas > 1 ? static_cast<int>(cluster.block_rank()) : 0;
  const int r = blockIdx.x / n_ctas;
  const int first = min(rank * slice, a.vocab), n = min(slice, a.vocab - first);
  if (n_ctas > 1) cluster_arrive_release();              // (waited for below: no CTA writes to one that is not there)
  griddep_wait();
  const T* in = static_cast<const T*>(a.x) + r * a.ld + first;
  float* out = a.out + r * a.ld_out + first;
  float temp = a.temperature ? a.temperature[r] : a.temperature_all;
  float top_p = 1.f;
  int top_k = 0;
  if (CUTS) {
    top_p = a.top_p ? a.top_p[r] : a.top_p_all;
    const int k = a.top_k ? a.top_k[r] : a.top_k_all;
    top_k = k > 0 && k < a.vocab ? k : 0;
  }
  bool bad = temp != temp || top_p != top_p;
  if (!(temp > 0.f)) temp = 0.f;
  top_p = top_p != top_p ? 1.f : fmaxf(top_p, 0.f);
  if (tid == 0) {
    s.slope = slope_of(temp);
    s.n_list[0] = s.n_list[1] = 0;
  }
  if (CUTS && tid >= 64 && tid < 64 + 33) s.exp2_of[tid - 64] = kExp2[tid - 64];

  constexpr int kFly = 16;
  float m = -INFINITY;
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
      m = fmaxf(m, v[j]);
      if (i < n) x[i] = v[j];
    }
  }
  m = warp_max(m);
  if (lane == 0) s.red[warp] = m;
  if (__syncthreads_or(bad) && tid == 0) flag_status(a.status, DVI_DEV_NONFINITE);
  m = warp_max(lane < kWarps ? s.red[lane] : -INFINITY);
  const Slope c = s.slope;

  // this CTA's sum of w (to its own maximum) or, for a greedy row, its first largest token
  float sum = 0.f;
  int at = 0x7fffffff;
  if (temp > 0.f) {
    if (m > -INFINITY) {
      for (int i = tid; i < n; i += kThreads) {
        const float w = weight(x[i], m, c);
        sum += w;
        if (!CUTS) x[i] = w;
      }
    }
    sum = warp_sum(sum);
    if (lane == 0) s.sum[warp] = sum;
  } else {
    for (int i = n - 1 - tid; i >= 0; i -= kThreads)
      if (x[i] == m) at = i;
    at = __reduce_min_sync(0xffffffffu, at);
    if (lane == 0) s.first[warp] = at;
  }
  __syncthreads();
  if (warp == 0) {
    if (n_ctas > 1) cluster_wait_acquire();
    sum = warp_sum(lane < kWarps && temp > 0.f ? s.sum[lane] : 0.f);
    at = __reduce_min_sync(0xffffffffu, lane < kWarps && !(temp > 0.f) ? s.first[lane] : 0x7fffffff);
    if (lane < n_ctas) {
      float2* p = n_ctas > 1 ? cluster.map_shared_rank(&s.peer[rank], lane) : &s.peer[0];
      int* f = n_ctas > 1 ? cluster.map_shared_rank(&s.peer_first[rank], lane) : &s.peer_first[0];
      *p = make_float2(m, sum);
      *f = at;
    }
  } else if (n_ctas > 1) {
    cluster_wait_acquire();
  }
  cluster_barrier(n_ctas);
  const float own = m;
  for (int q = 0; q < n_ctas; ++q) m = fmaxf(m, s.peer[q].x);

  if (!(temp > 0.f) || m == -INFINITY) {
    int q = 0;
    while (s.peer[q].x != m) ++q;
    const int hot = m > -INFINITY && q == rank ? s.peer_first[q] : -1;
    for (int i = tid; i < n; i += kThreads) out[i] = i == hot ? 1.f : 0.f;
    return;
  }
  sum = 0.f;
  for (int q = 0; q < n_ctas; ++q)
    if (s.peer[q].x > -INFINITY) sum += s.peer[q].y * weight(s.peer[q].x, m, c);
  if (!CUTS) {
    const float scale = own > -INFINITY ? weight(own, m, c) / sum : 0.f;
    for (int i = tid; i < n; i += kThreads) out[i] = own > -INFINITY ? x[i] * scale : 0.f;
    return;
  }
  unsigned long long upto = ~0ull;
  float inv = 1.f / sum;
  const RowState row = {x, first, n, m, ord(m), c};
  if (top_k || top_p < 1.f) {
    unsigned long long kept = 0, all = 0;
    if (top_k) upto = last_kept<false>(row, top_k, ~0ull, 0.f, n_ctas, h, s, &kept);
    for (int i = tid; i < n; i += kThreads)
      if (upto == ~0ull || row.place(x[i], i) <= upto) all += mass(x[i], m, c, s.exp2_of);
    kept = all = cluster_sum(all, 0, n_ctas, s);
    if (top_p < 1.f) {
      // tokens below (1 - p) S / V sum to less than the rest may, so the last kept one is
      // above that (S by the f32 sum is not less than what top_k leaves; half of it, for
      // its rounding)
      const float least = upto == ~0ull ? 0.5f * (1.f - top_p) * sum / static_cast<float>(a.vocab) : 0.f;
      const unsigned long long e = last_kept<true>(row, share_of(top_p, all), upto, least, n_ctas, h, s, &kept);
      if (e != ~0ull) upto = e;
      else kept = all;
    }
    inv = 1.f / (__ull2float_rn(kept) * 0x1p-44f);
  }
  const float x_cut = upto == ~0ull ? -INFINITY : from_ord(row.top - static_cast<uint32_t>(upto >> kIndexBits));
  const int i_cut = static_cast<int>(upto & ((1u << kIndexBits) - 1)) - first;
  for (int i = tid; i < n; i += kThreads) {
    const float v = x[i];
    const bool in_it = v > x_cut || (v == x_cut && i <= i_cut && v > -INFINITY);
    out[i] = in_it ? weight(v, m, c) * inv : 0.f;
  }
  // no CTA leaves while another may read what it found
  if (top_k || top_p < 1.f) cluster_barrier(n_ctas);
}

constexpr int kSlice = 16384;   // logits of a CTA where its row may have up to kMaxCtas: two CTAs an SM

template <typename T, bool CUTS>
cudaError_t launch(const TokenProbsArgs& a, cudaStream_t s) {
  auto kern = token_probs_kernel<T, CUTS>;
  static PerDevice per_device;
  per_device.once([&] {
    cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize,
                         kMaxVocab / kMaxCtas * static_cast<int>(sizeof(float)) + static_cast<int>(sizeof(Cuts)));
  });
  int ctas = 1;
  while (ctas < kMaxCtas && (ctas * kSlice < a.vocab || (static_cast<int64_t>(a.n_rows) * ctas < 152 && a.vocab / ctas > 4096)))
    ctas *= 2;
  if (static_cast<int64_t>(a.n_rows) * ctas > 0x7fffffffll) return cudaErrorInvalidConfiguration;
  const int slice = (a.vocab + ctas - 1) / ctas;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(a.n_rows) * ctas);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = (slice * sizeof(float) + 15) / 16 * 16 + (CUTS ? sizeof(Cuts) : 0);
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

}  // namespace

cudaError_t launch_token_probs(const TokenProbsArgs& a, int dtype, cudaStream_t s) {
  const bool cuts = a.top_k || a.top_p || a.top_p_all < 1.f || (a.top_k_all > 0 && a.top_k_all < a.vocab);
  if (dtype == DVI_BF16) return cuts ? launch<__nv_bfloat16, true>(a, s) : launch<__nv_bfloat16, false>(a, s);
  return cuts ? launch<float, true>(a, s) : launch<float, false>(a, s);
}

}  // namespace dvi
