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

// 2^(k / 32), k = 0 .. 31, as f32 pairs hi + lo.
__constant__ float2 kExp2[32] = {
    {0x1p+0f, 0.f}, {0x1.059b0ep+0f, -0x1.9d4f52p-25f}, {0x1.0b5586p+0f, 0x1.9f3122p-25f}, {0x1.11301ep+0f, -0x1.fdb496p-25f},
    {0x1.172b84p+0f, -0x1.c15742p-27f}, {0x1.1d4874p+0f, -0x1.d2e8cap-25f}, {0x1.2387a6p+0f, 0x1.ceac48p-25f}, {0x1.29e9ep+0f, -0x1.5c0424p-25f},
    {0x1.306fep+0f, 0x1.4636e2p-25f}, {0x1.371a74p+0f, -0x1.18aac6p-25f}, {0x1.3dea64p+0f, 0x1.824684p-25f}, {0x1.44e086p+0f, 0x1.8624b4p-30f},
    {0x1.4bfdaep+0f, -0x1.593abcp-25f}, {0x1.5342b6p+0f, -0x1.2c561p-25f}, {0x1.5ab07ep+0f, -0x1.5bd5ecp-27f}, {0x1.6247ecp+0f, -0x1.f8b55p-25f},
    {0x1.6a09e6p+0f, 0x1.9fcef4p-26f}, {0x1.71f75ep+0f, 0x1.1d8beep-25f}, {0x1.7a1148p+0f, -0x1.829fdp-25f}, {0x1.82589ap+0f, -0x1.accc7cp-26f},
    {0x1.8ace54p+0f, 0x1.15506ep-27f}, {0x1.93737cp+0f, -0x1.e64744p-25f}, {0x1.9c4918p+0f, 0x1.51f848p-27f}, {0x1.a5503cp+0f, -0x1.b83b54p-25f},
    {0x1.ae89fap+0f, -0x1.a94b14p-26f}, {0x1.b7f77p+0f, -0x1.a09438p-25f}, {0x1.c199bep+0f, -0x1.3d56b2p-27f}, {0x1.cb720ep+0f, -0x1.8837ccp-27f},
    {0x1.d5818ep+0f, -0x1.822dbcp-27f}, {0x1.dfc974p+0f, -0x1.908c94p-25f}, {0x1.ea4afap+0f, 0x1.52486cp-27f}, {0x1.f50766p+0f, -0x1.246ebp-26f}};

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

// Two f32 numbers in one register pair: an operation on both is one instruction.
struct Two {
  unsigned long long v;
};
__device__ __forceinline__ Two two(float a, float b) {
  Two r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ Two two(float a) { return two(a, a); }
__device__ __forceinline__ float2 split(Two a) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(a.v));
  return r;
}
__device__ __forceinline__ Two operator+(Two a, Two b) {
  Two r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
  return r;
}
__device__ __forceinline__ Two operator*(Two a, Two b) {
  Two r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
  return r;
}
__device__ __forceinline__ Two fma2(Two a, Two b, Two c) {
  Two r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
  return r;
}
__device__ __forceinline__ Two operator-(Two a, Two b) { return fma2(b, two(-1.f), a); }   // (the product is exact)

// w of two logits in units of 2^-44, off by about 2^-38; 0 below 2^-46.  x - m and its
// product t with the slope are f32 pairs; t = q / 32 + r, 2^(q / 32) comes from the table and an
// exponent, and 2^r = e^z = 1 + z + z^2 (1/2 + z/6 + z^2/24 + z^3/120) with |z| <= ln 2 / 64, of
// which only 1 + z needs the second number.  Adding 1.5 * 2^23 rounds to whole numbers and leaves
// them in the low bits.
struct Masses {
  unsigned long long a, b;
};
__device__ __forceinline__ Masses mass2(float xa, float xb, float m, Slope c, const float2* exp2_of) {
  const float kRound = 12582912.f, kLn2 = 0x1.62e430p-1f, kLn2Lo = -0x1.05c610p-29f;
  const Two x = two(xa, xb), top = two(m), ch = two(c.hi);
  const Two dh = x - top, back = dh - x;
  const Two dl = (x - (dh - back)) - (top + back);
  const Two th = dh * ch;
  const Two tl = fma2(dh, two(c.lo), fma2(dl, ch, fma2(dh, ch, two(0.f) - th)));
  const Two q = fma2(th, two(32.f), two(kRound)), r = fma2(q - two(kRound), two(-0.03125f), th);
  const Two z = r * two(kLn2);
  const Two zl = fma2(tl, two(kLn2), fma2(r, two(kLn2Lo), fma2(r, two(kLn2), two(0.f) - z)));
  const Two poly = fma2(z, fma2(z, fma2(z, two(1.f / 120.f), two(1.f / 24.f)), two(1.f / 6.f)), two(0.5f));
  const Two zz = z * z * poly;
  const Two p = z + zz, pl = ((z - p) + zz) + fma2(z, zl, zl);
  const float2 qs = split(q), ts = split(th);
  const int qa = __float_as_int(qs.x), qb = __float_as_int(qs.y);
  const float2 ta = exp2_of[qa & 31], tb = exp2_of[qb & 31];
  const Two t = two(ta.x, tb.x), prod = t * p;
  const Two e = fma2(t, p, two(0.f) - prod) + fma2(t, pl, two(ta.y, tb.y));
  const Two hi = t + prod, lo = ((t - hi) + prod) + e;
  // times 2^(n + 22), n = q >> 5 (the shift drops what 1.5 * 2^23 leaves above it): 22 bits, then
  // 22 more of what they leave
  const Two scale = two(__int_as_float(((qa >> 5) << 23) + ((22 + 127) << 23)),
                        __int_as_float(((qb >> 5) << 23) + ((22 + 127) << 23)));
  const Two h = hi * scale, u = h + two(kRound);
  const Two rest = fma2(lo, scale, h - (u - two(kRound)));
  const Two f = fma2(rest, two(4194304.f), two(kRound));
  const float2 us = split(u), fs = split(f);
  const int kBits = 0x4b400000;   // of 1.5 * 2^23
  const long long wa = static_cast<long long>(__float_as_int(us.x) - kBits) * 4194304 + (__float_as_int(fs.x) - kBits);
  const long long wb = static_cast<long long>(__float_as_int(us.y) - kBits) * 4194304 + (__float_as_int(fs.y) - kBits);
  return {ts.x > -46.f ? static_cast<unsigned long long>(wa) : 0ull,
          ts.y > -46.f ? static_cast<unsigned long long>(wb) : 0ull};
}
__device__ __noinline__ unsigned long long mass(float x, float m, Slope c, const float2* exp2_of) {
  return mass2(x, x, m, c, exp2_of).a;
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
  float2 exp2_of[32];
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
  int first, n;         // (n: up to a multiple of 4, with -inf behind the last token)
  float m;              // the row's maximum
  uint32_t top;         // ord(m)
  Slope c;
  __device__ __forceinline__ unsigned long long place(float v, int i) const {
    return (static_cast<unsigned long long>(top - ord(v + 0.f)) << kIndexBits) | static_cast<unsigned>(first + i);
  }
  __device__ __forceinline__ float logit(unsigned long long place) const {
    return from_ord(top - static_cast<uint32_t>(place >> kIndexBits));
  }
  __device__ __forceinline__ int bin(float v) const {   // (rounded by adding 1.5 * 2^23)
    const float t = __fmul_rn(__fmul_rn(__fsub_rn(m, v), c.hi), kBinsPerOctave);
    return __float_as_int(__fadd_rn(fminf(t, static_cast<float>(kBins - 1)), 12582912.f)) & 0xffff;
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
  uint2 lo[kMaxCtas], hi[kMaxCtas];
#pragma unroll
  for (int r = 0; r < kMaxCtas; ++r) {   // (all in flight)
    lo[r] = hi[r] = make_uint2(0, 0);
    if (r0 + r < r1) {
      lo[r] = reinterpret_cast<const uint2*>(cluster.map_shared_rank(h.lo, r0 + r))[tid];
      hi[r] = reinterpret_cast<const uint2*>(cluster.map_shared_rank(h.hi, r0 + r))[tid];
    }
  }
#pragma unroll
  for (int r = 0; r < kMaxCtas; ++r) {
    v[0] += (static_cast<unsigned long long>(hi[r].x) << 32) + lo[r].x;
    v[1] += (static_cast<unsigned long long>(hi[r].y) << 32) + lo[r].y;
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

// Tokens of the order up to one of them (all: those above -inf).
struct Upto {
  float x;
  int i;
  __device__ __forceinline__ bool has(float v, int at) const { return v > x || (v == x && at <= i); }
};

// The last kept token among those up to `upto`: before it the counts sum to less than top_k, or
// (MASS) the masses to less than top_p of all.  Returns the tokens up to it.  *kept: their sum.
// Tokens below `least` are known to be cut.  mine: the largest of the thread's own logits.
template <bool MASS>
__device__ Upto last_kept(const RowState& row, int top_k, float top_p, Upto upto, float least, float mine, int rank,
                          int n_ctas, Cuts& h, Small& s, unsigned long long* kept) {
  cg::cluster_group cluster = cg::this_cluster();
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const float4* x4 = reinterpret_cast<const float4*>(row.x);
  const int n4 = row.n / 4;
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
  if (MASS) {
    // (a mass is 0 below 2^-46)
    const float some = row.m - 46.f / row.c.hi * 1.0001f;
    unsigned long long all = 0;
    for (int g0 = warp * 32; g0 < n4; g0 += kThreads) {
      const int g = g0 + lane;
      float v[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
      if (g < n4) *reinterpret_cast<float4*>(v) = x4[g];
      bool in[4], any = false;
#pragma unroll
      for (int e = 0; e < 4; ++e) any |= in[e] = v[e] >= some && upto.has(v[e], 4 * g + e);
      if (!__any_sync(0xffffffffu, any)) continue;
#pragma unroll
      for (int e = 0; e < 4; e += 2) {
        const Masses w = mass2(v[e], v[e + 1], row.m, row.c, s.exp2_of);
        if (in[e] && w.a) {
          all += w.a;
          if (v[e] >= least) add_to_bin(h, row.bin(v[e]), w.a);
        }
        if (in[e + 1] && w.b) {
          all += w.b;
          if (v[e + 1] >= least) add_to_bin(h, row.bin(v[e + 1]), w.b);
        }
      }
    }
    give_sum(all, 1, rank, n_ctas, s);
  } else {
    for (int g = tid; g < n4; g += kThreads) {
      const float4 q = x4[g];
      const float v[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int bin = row.bin(v[e]);
        if (bin <= most && v[e] > -INFINITY) atomicAdd(&h.lo[bin], 1u);
      }
    }
  }
  cluster_barrier(n_ctas);
  unsigned long long target = top_k;
  if (MASS) {
    *kept = given_sum(1, n_ctas, s);
    target = share_of(top_p, *kept);
  }
  const int bin = find_bin(0, target, 0, n_ctas, h, s, &before);
  if (bin < 0) return upto;
  int& found = s.n_list[MASS];
  auto counts = [&](float v, int i) { return v >= least && v > -INFINITY && upto.has(v, i); };
  for (int g = tid; g < n4; g += kThreads) {
    const float4 q = x4[g];
    const float v[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (row.bin(v[e]) != bin || !counts(v[e], 4 * g + e)) continue;
      const int at = atomicAdd(&found, 1);
      if (at < kList) h.list[at] = row.place(v[e], 4 * g + e);
    }
  }
  cluster_barrier(n_ctas);
  // how many each CTA has found, a lane a CTA; the warps share the CTAs' lists
  const int there = lane < n_ctas ? *cluster.map_shared_rank(&found, lane) : 0;
  int upto_here = there;
#pragma unroll
  for (int o = 1; o < kMaxCtas; o <<= 1) {
    const int w = __shfl_up_sync(0xffffffffu, upto_here, o);
    if (lane >= o) upto_here += w;
  }
  const int n = __shfl_sync(0xffffffffu, upto_here, kMaxCtas - 1);
  unsigned long long cut;
  if (n <= kList) {
    const int per = kWarps / n_ctas, from = warp / per;
    const int m = __shfl_sync(0xffffffffu, there, from), at = __shfl_sync(0xffffffffu, upto_here, from) - m;
    const unsigned long long* list = cluster.map_shared_rank(h.list, from);
    for (int i = warp % per * 32 + lane; i < m; i += per * 32) {
      const unsigned long long p = list[i];
      h.key[at + i] = p;
      if (MASS) h.mass[at + i] = mass(row.logit(p), row.m, row.c, s.exp2_of);
    }
    __syncthreads();
    cut = last_of_list<MASS>(n, before, target, rank, h, s, kept);
  } else {
    before = cut = 0;
    for (int shift = 32 + kIndexBits - kBinBits;; shift = shift > kBinBits ? shift - kBinBits : 0) {
      clear_bins(h);
      for (int i = tid; i < row.n; i += kThreads) {
        const float x = row.x[i];
        if (!counts(x, i)) continue;
        const unsigned long long p = row.place(x, i);
        if (p < cut || ((p - cut) >> shift) >= kBins) continue;
        add_to_bin(h, static_cast<int>((p - cut) >> shift), MASS ? mass(x, row.m, row.c, s.exp2_of) : 1ull);
      }
      cluster_barrier(n_ctas);
      const int b = find_bin(before, target, 0, n_ctas, h, s, &before);   // (found: the sums are those of the first bins)
      cut += static_cast<unsigned long long>(b) << shift;
      if (shift == 0) {
        // one token a bin
        *kept = before;
        for (int r = 0; r < n_ctas; ++r)
          *kept += (static_cast<unsigned long long>(cluster.map_shared_rank(h.hi, r)[b]) << 32) +
                   cluster.map_shared_rank(h.lo, r)[b];
      }
      cluster_barrier(n_ctas);   // before the bins are cleared
      if (shift == 0) break;
    }
  }
  return {row.logit(cut), static_cast<int>(cut & ((1u << kIndexBits) - 1)) - row.first};
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
template <int WARPS>
__device__ __forceinline__ void join(const float2* peer, int n_ctas, bool greedy, Slope c, float* m, float* sum, int* hot) {
  const int lane = threadIdx.x & 31;
  float top = -INFINITY;
  for (int i = lane; i < n_ctas * WARPS; i += 32) top = fmaxf(top, peer[i].x);
  top = warp_max(top);
  float all = 0.f;
  int first = 0x7fffffff;
  for (int i = lane; i < n_ctas * WARPS; i += 32) {
    const float2 p = peer[i];
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

// The CTA's own first arrival at the cluster's barrier, which only says that it is there.
__device__ __forceinline__ void cluster_hello(int n_ctas) {
  if (n_ctas > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
}

// Four logits that lie together.
__device__ __forceinline__ float4 load4(const float* p) { return *reinterpret_cast<const float4*>(p); }
__device__ __forceinline__ float4 load4(const __nv_bfloat16* p) {
  const uint2 w = *reinterpret_cast<const uint2*>(p);
  return make_float4(bf16_lo(w.x), bf16_hi(w.x), bf16_lo(w.y), bf16_hi(w.y));
}

// Rows without cuts: NV logits a thread, in registers; four at a time that lie together (V4)
// or one.  A warp takes w to its own maximum.
template <typename T, int NV, int THREADS, bool V4>
__global__ void __launch_bounds__(THREADS, 32768 / (NV * THREADS))
    token_probs_kernel(TokenProbsArgs a, int n_ctas, int slice) {
  __shared__ float2 peer[kMaxCtas * THREADS / 32];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int rank = n_ctas > 1 ? static_cast<int>(cg::this_cluster().block_rank()) : 0;
  const int r = blockIdx.x / n_ctas;
  const int first = min(rank * slice, a.vocab), n = min(slice, a.vocab - first);
  cluster_hello(n_ctas);                                 // (waited for below: no CTA writes to one that is not there)
  griddep_wait();
  const T* in = static_cast<const T*>(a.x) + r * a.ld + first;
  float* out = a.out + r * a.ld_out + first;
  auto index = [&](int j) { return V4 ? ((j >> 2) * THREADS + tid) * 4 + (j & 3) : j * THREADS + tid; };
  float v[NV];
  if (V4) {
#pragma unroll
    for (int j = 0; j < NV; j += 4) {
      const int i = index(j);
      float4 q = make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
      if (i + 4 <= n) {
        q = load4(in + i);
      } else if (i < n) {
        q.x = DT<T>::ld(in + i);
        if (i + 1 < n) q.y = DT<T>::ld(in + i + 1);
        if (i + 2 < n) q.z = DT<T>::ld(in + i + 2);
      }
      v[j] = q.x, v[j + 1] = q.y, v[j + 2] = q.z, v[j + 3] = q.w;
    }
  } else {
#pragma unroll
    for (int j = 0; j < NV; ++j) v[j] = index(j) < n ? DT<T>::ld(in + index(j)) : -INFINITY;
  }
  const Settings set(a, r);
  const bool greedy = set.temperature == 0.f;
  const Slope c = {__fdiv_rn(1.44269504f, fminf(fmaxf(set.temperature, 0x1p-100f), 0x1p100f)), 0.f};
  bool bad = set.bad;
  float m = -INFINITY, odd = 0.f;   // odd: 0 of finite logits
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    m = fmaxf(m, v[j]);
    odd = fmaf(v[j], 0.f, odd);
  }
  if (__any_sync(0xffffffffu, odd != 0.f)) {
    // (masked tokens, too, and what is behind the row's end)
    m = -INFINITY;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      bad |= !(v[j] < INFINITY);
      v[j] = clean(v[j]);
      m = fmaxf(m, v[j]);
    }
  }
  m = warp_max(m);
  float2 mine = make_float2(m, 0.f);
  float back = 1.f;
  if (greedy) {
    int at = 0x7fffffff;
#pragma unroll
    for (int j = NV - 1; j >= 0; --j)
      if (v[j] == m) at = first + index(j);
    mine.y = __int_as_float(__reduce_min_sync(0xffffffffu, at));
  } else if (m > -INFINITY) {
    // x c - m c in one step where m c is small enough for its rounding to be taken back
    const float mc = m * c.hi;
    float sum[4] = {0.f, 0.f, 0.f, 0.f};
    if (fabsf(mc) <= 0x1p20f) {
      back = exp2f(-fmaf(m, c.hi, -mc));
#pragma unroll
      for (int j = 0; j < NV; ++j) sum[j & 3] += v[j] = exp2f(fmaf(v[j], c.hi, -mc));
    } else {
#pragma unroll
      for (int j = 0; j < NV; ++j) sum[j & 3] += v[j] = weight(v[j], m, c);
    }
    mine.y = warp_sum((sum[0] + sum[1]) + (sum[2] + sum[3])) * back;
  }
  if (bad) flag_status(a.status, DVI_DEV_NONFINITE);
  if (n_ctas > 1) {
    cluster_wait_acquire();
    if (lane < n_ctas) *cg::this_cluster().map_shared_rank(&peer[rank * THREADS / 32 + warp], lane) = mine;
  } else if (lane == 0) {
    peer[warp] = mine;
  }
  cluster_barrier(n_ctas);
  float top, sum;
  int hot;
  join<THREADS / 32>(peer, n_ctas, greedy, c, &top, &sum, &hot);
  float scale = 0.f;
  if (greedy) {
#pragma unroll
    for (int j = 0; j < NV; ++j) v[j] = top > -INFINITY && first + index(j) == hot ? 1.f : 0.f;
    scale = 1.f;
  } else if (m > -INFINITY) {
    scale = weight(m, top, c) * back / sum;
  } else {
#pragma unroll
    for (int j = 0; j < NV; ++j) v[j] = 0.f;
  }
  if (V4) {
#pragma unroll
    for (int j = 0; j < NV; j += 4) {
      const int i = index(j);
      if (i + 4 <= n) {
        *reinterpret_cast<float4*>(out + i) =
            make_float4(v[j] * scale, v[j + 1] * scale, v[j + 2] * scale, v[j + 3] * scale);
      } else if (i < n) {
        out[i] = v[j] * scale;
        if (i + 1 < n) out[i + 1] = v[j + 1] * scale;
        if (i + 2 < n) out[i + 2] = v[j + 2] * scale;
      }
    }
  } else {
#pragma unroll
    for (int j = 0; j < NV; ++j)
      if (index(j) < n) out[index(j)] = v[j] * scale;
  }
}

// Rows with cuts: a slice in shared memory.
template <typename T, bool V4>
__global__ void __launch_bounds__(kThreads, 2) token_probs_cut_kernel(TokenProbsArgs a, int n_ctas, int slice) {
  extern __shared__ __align__(16) unsigned char dynamic[];
  __shared__ Small s;
  Cuts& h = *reinterpret_cast<Cuts*>(dynamic);
  float* x = reinterpret_cast<float*>(dynamic + sizeof(Cuts));
  float4* x4 = reinterpret_cast<float4*>(x);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int rank = n_ctas > 1 ? static_cast<int>(cg::this_cluster().block_rank()) : 0;
  const int r = blockIdx.x / n_ctas;
  const int first = min(rank * slice, a.vocab), n = min(slice, a.vocab - first), n4 = (n + 3) / 4;
  cluster_hello(n_ctas);
  griddep_wait();
  const T* in = static_cast<const T*>(a.x) + r * a.ld + first;
  float* out = a.out + r * a.ld_out + first;
  const Settings set(a, r);
  const bool greedy = set.temperature == 0.f;
  if (tid == 0) {
    s.slope = slope_of(set.temperature);
    s.n_list[0] = s.n_list[1] = 0;
  }
  if (tid >= 64 && tid < 64 + 32) s.exp2_of[tid - 64] = kExp2[tid - 64];

  float own = -INFINITY, odd = 0.f;   // odd: 0 of finite logits
  constexpr int kFly = 16;
  if (V4) {
    for (int g0 = 0; g0 < n4; g0 += kFly / 4 * kThreads) {
      float4 q[kFly / 4];
#pragma unroll
      for (int j = 0; j < kFly / 4; ++j) {
        const int g = g0 + j * kThreads + tid, i = 4 * g;
        q[j] = make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
        if (i + 4 <= n) {
          q[j] = load4(in + i);
        } else if (i < n) {
          q[j].x = DT<T>::ld(in + i);
          if (i + 1 < n) q[j].y = DT<T>::ld(in + i + 1);
          if (i + 2 < n) q[j].z = DT<T>::ld(in + i + 2);
        }
      }
#pragma unroll
      for (int j = 0; j < kFly / 4; ++j) {
        const int g = g0 + j * kThreads + tid;
        if (g >= n4) continue;
        own = fmaxf(own, fmaxf(fmaxf(q[j].x, q[j].y), fmaxf(q[j].z, q[j].w)));
        odd = fmaf(q[j].x, 0.f, fmaf(q[j].y, 0.f, fmaf(q[j].z, 0.f, fmaf(q[j].w, 0.f, odd))));
        x4[g] = q[j];
      }
    }
  } else {
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
        own = fmaxf(own, v[j]);
        if (i < n) odd = fmaf(v[j], 0.f, odd);
        if (i < 4 * n4) x[i] = v[j];
      }
    }
  }
  // the tokens that the thread has loaded
  auto each = [&](auto f) {
    if (V4) {
      for (int g = tid; g < n4; g += kThreads)
        for (int i = 4 * g; i < 4 * g + 4; ++i) f(i);
    } else {
      for (int i = tid; i < n; i += kThreads) f(i);
    }
  };
  bool bad = set.bad;
  if (__syncthreads_or(odd != 0.f)) {
    // (masked tokens, too, and the -inf behind a row that ends within four)
    own = -INFINITY;
    each([&](int i) {
      bad |= !(x[i] < INFINITY);
      x[i] = clean(x[i]);
      own = fmaxf(own, x[i]);
    });
    __syncthreads();
  }
  if (bad) flag_status(a.status, DVI_DEV_NONFINITE);
  const float m = warp_max(own);
  const Slope c = s.slope;
  // (of the sum of w the largest logits of the threads: a lower bound is enough)
  float2 mine = make_float2(m, 0.f);
  if (greedy) {
    int at = 0x7fffffff;
    if (m > -INFINITY && own == m)
      each([&](int i) {
        if (x[i] == m) at = min(at, first + i);
      });
    mine.y = __int_as_float(__reduce_min_sync(0xffffffffu, at));
  } else if (m > -INFINITY) {
    mine.y = warp_sum(weight(own, m, c));
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
  join<kWarps>(s.peer, n_ctas, greedy, c, &top, &sum, &hot);
  if (greedy || top == -INFINITY) {
    for (int i = tid; i < n; i += kThreads) out[i] = top > -INFINITY && first + i == hot ? 1.f : 0.f;
    return;
  }
  const RowState row = {x, first, 4 * n4, top, ord(top + 0.f), c};
  Upto upto = {-INFINITY, 0x7fffffff};
  unsigned long long kept = 0;
  if (set.top_k) upto = last_kept<false>(row, set.top_k, 1.f, upto, -INFINITY, own, rank, n_ctas, h, s, &kept);
  if (set.top_p < 1.f) {
    // tokens below (1 - p) S / V sum to less than what may be cut, so the last kept one is
    // above that (half of it, for the sum's rounding)
    float least = -INFINITY;
    if (upto.x == -INFINITY)
      least = top + log2f(0.5f * (1.f - set.top_p) * sum / static_cast<float>(a.vocab)) / c.hi * 1.0001f;
    upto = last_kept<true>(row, 0, set.top_p, upto, least, own, rank, n_ctas, h, s, &kept);
  } else {
    unsigned long long all = 0;
    for (int i = tid; i < n; i += kThreads)
      if (upto.has(x[i], i)) all += mass(x[i], top, c, s.exp2_of);
    give_sum(all, 0, rank, n_ctas, s);
    cluster_barrier(n_ctas);
    kept = given_sum(0, n_ctas, s);
  }
  if (n_ctas > 1) cluster_arrive_release();   // nothing of the others is read from here on
  const float inv = 1.f / (__ull2float_rn(kept) * 0x1p-44f);
  auto prob = [&](float v, int i) { return upto.has(v, i) ? weight(v, top, c) * inv : 0.f; };
  if (V4) {
    for (int g = tid; g < n4; g += kThreads) {
      const float4 q = x4[g];
      const int i = 4 * g;
      const float4 p = make_float4(prob(q.x, i), prob(q.y, i + 1), prob(q.z, i + 2), prob(q.w, i + 3));
      if (i + 4 <= n) {
        *reinterpret_cast<float4*>(out + i) = p;
      } else {
        out[i] = p.x;
        if (i + 1 < n) out[i + 1] = p.y;
        if (i + 2 < n) out[i + 2] = p.z;
      }
    }
  } else {
    for (int i = tid; i < n; i += kThreads) out[i] = prob(x[i], i);
  }
  if (n_ctas > 1) cluster_wait_acquire();     // (and no CTA leaves while another may read what it found)
}

template <typename K>
cudaError_t launch(K kern, const TokenProbsArgs& a, int ctas, int threads, size_t smem, cudaStream_t s) {
  if (static_cast<int64_t>(a.n_rows) * ctas > 0x7fffffffll) return cudaErrorInvalidConfiguration;
  const int slice = ((a.vocab + ctas - 1) / ctas + 3) / 4 * 4;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(a.n_rows) * ctas);
  cfg.blockDim = dim3(threads);
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

// Whether rows start on the boundaries of four elements of both sides.
template <typename T>
bool fours(const TokenProbsArgs& a) {
  return reinterpret_cast<uintptr_t>(a.x) % (4 * sizeof(T)) == 0 && reinterpret_cast<uintptr_t>(a.out) % 16 == 0 &&
         (a.n_rows == 1 || (a.ld % 4 == 0 && a.ld_out % 4 == 0));
}

template <typename T, bool V4>
cudaError_t launch_plain(const TokenProbsArgs& a, cudaStream_t s) {
  const int most = a.vocab <= 32 * 256 * kMaxCtas ? 32 * 256 : a.vocab <= 32 * 512 * kMaxCtas ? 32 * 512 : 64 * 512;
  int ctas = 1;
  while (ctas * most < a.vocab) ctas *= 2;
  if (most == 32 * 256) return launch(token_probs_kernel<T, 32, 256, V4>, a, ctas, 256, 0, s);
  return most == 32 * 512 ? launch(token_probs_kernel<T, 32, 512, V4>, a, ctas, 512, 0, s)
                          : launch(token_probs_kernel<T, 64, 512, V4>, a, ctas, 512, 0, s);
}
template <typename T>
cudaError_t launch_plain(const TokenProbsArgs& a, cudaStream_t s) {
  return fours<T>(a) ? launch_plain<T, true>(a, s) : launch_plain<T, false>(a, s);
}

constexpr int kSlice = 16384;   // logits of a CTA where its row may have up to kMaxCtas: two CTAs an SM

template <typename T, bool V4>
cudaError_t launch_cut(const TokenProbsArgs& a, cudaStream_t s) {
  static PerDevice per_device;
  per_device.once([&] {
    cudaFuncSetAttribute(token_probs_cut_kernel<T, V4>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                         kMaxVocab / kMaxCtas * static_cast<int>(sizeof(float)) + static_cast<int>(sizeof(Cuts)));
  });
  int ctas = 1;
  while (ctas < kMaxCtas && (ctas * kSlice < a.vocab || (static_cast<int64_t>(a.n_rows) * ctas < 152 && a.vocab / ctas > 4096)))
    ctas *= 2;
  return launch(token_probs_cut_kernel<T, V4>, a, ctas, kThreads, sizeof(Cuts), s);
}
template <typename T>
cudaError_t launch_cut(const TokenProbsArgs& a, cudaStream_t s) {
  return fours<T>(a) ? launch_cut<T, true>(a, s) : launch_cut<T, false>(a, s);
}

}  // namespace

cudaError_t launch_token_probs(const TokenProbsArgs& a, int dtype, cudaStream_t s) {
  const bool cuts = a.top_k || a.top_p || a.top_p_all < 1.f || (a.top_k_all > 0 && a.top_k_all < a.vocab);
  if (dtype == DVI_BF16) return cuts ? launch_cut<__nv_bfloat16>(a, s) : launch_plain<__nv_bfloat16>(a, s);
  return cuts ? launch_cut<float>(a, s) : launch_plain<float>(a, s);
}

}  // namespace dvi
