// Probabilities of sampling from logits: temperature, top-k, top-p.
//
// With tokens in the order of their logits (equal ones by index) and w =
// exp((x - max) / T), a row's kept tokens are a prefix of the order; the prefix
// ends at the last token whose rank is below top_k and before which the sum of
// w is below top_p of the whole.  That token is found by its place in the order
// as a number, (ord(max) - ord(x)) << 18 | index: 11 bits of it at a time, by
// histograms of counts and of w.  Sums of w are whole numbers, so they do not
// depend on the order of the atomics.
#include <cooperative_groups.h>

#include "sample.cuh"

namespace dvi {
namespace {

constexpr int kThreads = 512;
constexpr int kBins = 2048;
constexpr int kBinBits = 11;
constexpr int kIndexBits = 18;                   // kMaxVocab
constexpr int kPer = kBins / kThreads;
constexpr unsigned long long kOne = 1ull << 44;  // w = 1

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

// f32 as a number that grows with it.
__device__ __forceinline__ uint32_t ord(float x) {
  const uint32_t b = __float_as_uint(x);
  return (b & 0x80000000u) ? ~b : (b | 0x80000000u);
}

struct Shared {
  unsigned long long mass[kBins];
  unsigned count[kBins];
  float2 exp2_of[33];
  unsigned long long part[kThreads / 32];
  float red[kThreads / 32];
  int first;
  int found;
  unsigned long long excl, in_bin;
};

__device__ __forceinline__ unsigned long long warp_sum_u64(unsigned long long v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

template <typename T>
struct Row {
  const T* x;
  int V;
  __device__ __forceinline__ float at(int i) const {
    const float v = DT<T>::ld(x + i);
    // NaN as -inf; +inf as the largest number; -0 as 0
    return v != v ? -INFINITY : fminf(v, 3.402823466e38f) + 0.f;
  }
};

__device__ unsigned long long block_sum(unsigned long long v, Shared& s) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  v = warp_sum_u64(v);
  __syncthreads();
  if (lane == 0) s.part[warp] = v;
  __syncthreads();
  v = lane < kThreads / 32 ? s.part[lane] : 0;
  return warp_sum_u64(v);
}

// The place of the last kept token: before it the counts (or, over tokens up to
// `upto`, the masses) sum to less than target.  *kept: the sum up to it.  ~0 if
// the whole sum is less than target.
template <bool MASS, typename T>
__device__ unsigned long long last_kept(const Row<T>& row, float m, Slope c, unsigned long long target,
                                        unsigned long long upto, Shared& s, unsigned long long* kept) {
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t top = ord(m);
  unsigned long long lo = 0, before = 0;
  int shift = 32 + kIndexBits - kBinBits;
  for (;;) {
    __syncthreads();
    for (int i = tid; i < kBins; i += kThreads) s.mass[i] = 0, s.count[i] = 0;
    if (tid == 0) s.found = -1;
    __syncthreads();
    for (int i = tid; i < row.V; i += kThreads) {
      const float x = row.at(i);
      if (x == -INFINITY) continue;
      const unsigned long long d = (static_cast<unsigned long long>(top - ord(x)) << kIndexBits) | i;
      if (d < lo || d > upto || ((d - lo) >> shift) >= kBins) continue;
      const int bin = static_cast<int>((d - lo) >> shift);
      if (MASS)
        atomicAdd(&s.mass[bin], mass(x, m, c, s.exp2_of));
      else
        atomicAdd(&s.count[bin], 1u);
    }
    __syncthreads();
    unsigned long long v[kPer], sum = 0;
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      v[j] = MASS ? s.mass[tid * kPer + j] : s.count[tid * kPer + j];
      sum += v[j];
    }
    unsigned long long incl = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const unsigned long long w = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += w;
    }
    if (lane == 31) s.part[warp] = incl;
    __syncthreads();
    unsigned long long at = before + incl - sum;
    for (int w = 0; w < warp; ++w) at += s.part[w];
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      if (at < target && at + v[j] >= target) s.found = tid * kPer + j, s.excl = at, s.in_bin = v[j];
      at += v[j];
    }
    __syncthreads();
    if (s.found < 0) return ~0ull;
    before = s.excl;
    lo += static_cast<unsigned long long>(s.found) << shift;
    *kept = before + s.in_bin;
    if (shift == 0) return lo;
    shift = shift > kBinBits ? shift - kBinBits : 0;
  }
}

template <typename T>
__global__ void __launch_bounds__(kThreads) token_probs_kernel(TokenProbsArgs a) {
  __shared__ Shared s;
  griddep_wait();
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int r = blockIdx.x;
  const Row<T> row = {static_cast<const T*>(a.x) + r * a.ld, a.vocab};
  float* out = a.out + r * a.ld_out;
  float temp = a.temperature ? a.temperature[r] : a.temperature_all;
  float top_p = a.top_p ? a.top_p[r] : a.top_p_all;
  const int k_arg = a.top_k ? a.top_k[r] : a.top_k_all;
  bool bad = temp != temp || top_p != top_p;
  if (!(temp > 0.f)) temp = 0.f;
  if (top_p != top_p) top_p = 1.f;
  const int top_k = k_arg > 0 && k_arg < a.vocab ? k_arg : 0;
  if (tid < 33) s.exp2_of[tid] = kExp2[tid];
  if (tid == 0) s.first = a.vocab;

  float m = -INFINITY;
  for (int i = tid; i < a.vocab; i += kThreads) {
    const float raw = DT<T>::ld(row.x + i);
    bad |= raw != raw || raw == INFINITY;
    m = fmaxf(m, row.at(i));
  }
  m = warp_max(m);
  if (lane == 0) s.red[warp] = m;
  if (__syncthreads_or(bad) && tid == 0) flag_status(a.status, DVI_DEV_NONFINITE);
  m = warp_max(lane < kThreads / 32 ? s.red[lane] : -INFINITY);
  if (m == -INFINITY) {
    for (int i = tid; i < a.vocab; i += kThreads) out[i] = 0.f;
    return;
  }
  if (temp == 0.f) {
    int first = a.vocab;
    for (int i = tid; i < a.vocab; i += kThreads)
      if (row.at(i) == m) first = min(first, i);
    atomicMin(&s.first, first);
    __syncthreads();
    for (int i = tid; i < a.vocab; i += kThreads) out[i] = i == s.first ? 1.f : 0.f;
    return;
  }
  const Slope c = slope_of(temp);
  const uint32_t top = ord(m);
  unsigned long long upto = ~0ull, kept = 0;
  if (top_k) upto = last_kept<false>(row, m, c, top_k, ~0ull, s, &kept);
  unsigned long long sum = 0;
  for (int i = tid; i < a.vocab; i += kThreads) {
    const float x = row.at(i);
    if (((static_cast<unsigned long long>(top - ord(x)) << kIndexBits) | i) <= upto) sum += mass(x, m, c, s.exp2_of);
  }
  sum = block_sum(sum, s);
  if (top_p < 1.f) {
    const unsigned long long target = static_cast<unsigned long long>(ceil(static_cast<double>(top_p) * static_cast<double>(sum)));
    const unsigned long long e = last_kept<true>(row, m, c, target ? target : 1, upto, s, &kept);
    if (e != ~0ull) upto = e, sum = kept;
  }
  const float inv = static_cast<float>(static_cast<double>(kOne) / static_cast<double>(sum));
  for (int i = tid; i < a.vocab; i += kThreads) {
    const float x = row.at(i);
    const bool in = x != -INFINITY && ((static_cast<unsigned long long>(top - ord(x)) << kIndexBits) | i) <= upto;
    out[i] = in ? weight(x, m, c) * inv : 0.f;
  }
}

}  // namespace

cudaError_t launch_token_probs(const TokenProbsArgs& a, int dtype, cudaStream_t s) {
  auto kern = dtype == DVI_BF16 ? token_probs_kernel<__nv_bfloat16> : token_probs_kernel<float>;
  return launch_pdl(kern, dim3(a.n_rows), dim3(kThreads), 0, s, a);
}

}  // namespace dvi
