// Probabilities of sampling from logits with tokens cut off, for short rows: a CTA has a row in
// registers, a few logits a thread.
//
// The last kept token is looked for among the logits themselves: how many tokens, or how much of
// w, lies at or above the middle of what is left, until few are left, which are put in order.  That takes
// about log2 of the row's length less 5 turns of one barrier each, of which many CTAs share an SM; the
// histogram and the exchanges that longer rows need cost the same for a short one.
//
// Bound by that chain of turns: 576 rows of 1024 with the 50 likeliest 6.1 us, with top_p 7.8 (as longer rows 17.8
// and 17.7), 576 of 2048 10.5 and 14.4 (18.3 and 19.2); 576 of 4000 on 512 threads 21.5 and 32.4, where
// the histogram takes 20.4 and 25.6.
#include "token_mass.cuh"

namespace dvi {
namespace {

constexpr int kByValue = 16;   // turns by the logits' values, then at most 32
constexpr int kApart = 8;      // turns before it is looked at which tokens are left
constexpr int kFew = 32;       // tokens that are put in order at last

template <int THREADS>
struct Short {
  static constexpr int kWarps = THREADS / 32;
  float top[kWarps], low[kWarps];
  int first[kWarps];
  unsigned long long sum[2][kWarps];     // (in turns)
  unsigned count[2][kWarps];
  uint32_t least[2][kWarps], most[2][kWarps];
  unsigned n_few[2];                     // of the counts, of the masses
  ulonglong2 few[2][kFew];               // order and (turned round) index, mass; 0 behind them
};

__device__ __forceinline__ unsigned long long warp_total(unsigned long long v) {   // v below 2^52
  const unsigned a = __reduce_add_sync(0xffffffffu, static_cast<unsigned>(v) & 0x3ffffffu),
                 b = __reduce_add_sync(0xffffffffu, static_cast<unsigned>(v >> 26));
  return a + (static_cast<unsigned long long>(b) << 26);
}

// What there is of some tokens: how many, and their masses.
struct Part {
  unsigned count = 0;
  unsigned long long sum = 0;
};

// Sums over the CTA, one barrier each.
template <int THREADS>
struct Turns {
  static constexpr int kWarps = THREADS / 32;
  Short<THREADS>& s;
  int turn = 0;
  template <bool MASS>
  __device__ __forceinline__ void all(Part& p) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, t = turn++ & 1;
    p.count = __reduce_add_sync(0xffffffffu, p.count);
    if (MASS) p.sum = warp_total(p.sum);
    if (lane == 0) {
      s.count[t][warp] = p.count;
      if (MASS) s.sum[t][warp] = p.sum;
    }
    __syncthreads();
    p.count = 0, p.sum = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      p.count += s.count[t][w];
      if (MASS) p.sum += s.sum[t][w];
    }
  }
  // The least and the most.
  __device__ __forceinline__ void ends(uint32_t& least, uint32_t& most) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, t = turn++ & 1;
    least = __reduce_min_sync(0xffffffffu, least);
    most = __reduce_max_sync(0xffffffffu, most);
    if (lane == 0) s.least[t][warp] = least, s.most[t][warp] = most;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWarps; ++w) least = min(least, s.least[t][w]), most = max(most, s.most[t][w]);
  }
};

// Of the thread's tokens (o[j]: the logit's order, 0 of those that are out; token j * THREADS + tid) the last up to
// which those in order are target or more, or (MASS) their masses sum to it.  `whole` is what all are, target at
// least; orders are least to top.  Takes out (o[j] = 0) what is behind it, and returns the sum up to it.
template <bool MASS, int THREADS, int NV>
__device__ unsigned long long cut_after(uint32_t (&o)[NV], const unsigned long long (&mass)[NV], unsigned long long target,
                                        const Part& whole, uint32_t least, uint32_t top, Turns<THREADS>& turns) {
  const int tid = threadIdx.x, lane = tid & 31;
  Short<THREADS>& s = turns.s;
  // those at lo or above reach target, those at hi or above do not
  uint32_t lo = least, hi = top + 1;
  unsigned n_lo = whole.count, n_hi = 0;
  unsigned long long at_lo = MASS ? whole.sum : n_lo, at_hi = 0;
  for (int turn = 0; hi - lo > 1 && n_lo - n_hi > kFew; ++turn) {
    // the middle of the logits, or (where they differ by orders of magnitude) of their places in the order
    uint32_t mid = lo + (hi - lo) / 2;
    if (turn < kByValue) mid = min(max(ord(0.5f * from_ord(lo) + 0.5f * from_ord(hi - 1)), lo + 1), hi - 1);
    Part p;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      if (o[j] < mid) continue;
      ++p.count;
      if (MASS) p.sum += mass[j];
    }
    turns.template all<MASS>(p);
    const unsigned long long v = MASS ? p.sum : p.count;
    if (v >= target) lo = mid, n_lo = p.count, at_lo = v;
    else hi = mid, n_hi = p.count, at_hi = v;
    if (turn >= kApart && n_lo - n_hi > kFew) {
      // (equal ones among them, or far apart: on from token to token)
      uint32_t from = 0xffffffffu, to = 0;
#pragma unroll
      for (int j = 0; j < NV; ++j)
        if (o[j] >= lo && o[j] < hi) from = min(from, o[j]), to = max(to, o[j]);
      turns.ends(from, to);
      lo = from, hi = to + 1;
    }
  }
  uint32_t last = lo;
  int upto = 0x7fffffff;
  unsigned long long kept = at_lo;
  if (n_lo - n_hi <= kFew) {
    // a lane for each, in every warp
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      if (o[j] < lo || o[j] >= hi) continue;
      s.few[MASS][atomicAdd(&s.n_few[MASS], 1u)] =
          make_ulonglong2((static_cast<unsigned long long>(o[j]) << 32) | ~static_cast<unsigned>(j * THREADS + tid), MASS ? mass[j] : 1);
    }
    __syncthreads();
    const ulonglong2 mine = s.few[MASS][lane];
    unsigned long long before = at_hi;
#pragma unroll 8
    for (int i = 0; i < kFew; ++i) {
      const ulonglong2 other = s.few[MASS][i];
      if (other.x > mine.x) before += other.y;
    }
    const int from = __ffs(__ballot_sync(0xffffffffu, before < target && before + mine.y >= target)) - 1;
    const unsigned long long key = __shfl_sync(0xffffffffu, mine.x, from);
    last = static_cast<uint32_t>(key >> 32);
    upto = static_cast<int>(~static_cast<unsigned>(key));
    kept = __shfl_sync(0xffffffffu, before + mine.y, from);
  } else {
    // of those at lo, which are equal, the first so many by index
    const unsigned equal = n_lo - n_hi;
    const unsigned long long one = (at_lo - at_hi) / equal;
    const unsigned want = static_cast<unsigned>((target - at_hi + one - 1) / one);
    kept = at_hi + want * one;
    if (want < equal) {
      int a = -1, b = THREADS * NV - 1;   // up to a there are fewer than want, up to b there are not
      while (b - a > 1) {
        const int mid = (a + b) / 2;
        Part p;
#pragma unroll
        for (int j = 0; j < NV; ++j) p.count += o[j] == lo && j * THREADS + tid <= mid;
        turns.template all<false>(p);
        if (p.count >= want) b = mid;
        else a = mid;
      }
      upto = b;
    }
  }
#pragma unroll
  for (int j = 0; j < NV; ++j)
    if (o[j] < last || (o[j] == last && j * THREADS + tid > upto)) o[j] = 0;
  return kept;
}

template <typename T, int NV, int THREADS, int CTAS_AN_SM>
__global__ void __launch_bounds__(THREADS, CTAS_AN_SM) token_probs_short_kernel(TokenProbsArgs a) {
  __shared__ Short<THREADS> s;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, r = blockIdx.x, n = a.vocab;
  griddep_wait();
  const T* in = static_cast<const T*>(a.x) + r * a.ld;
  float* out = a.out + r * a.ld_out;
  float x[NV];
#pragma unroll
  for (int j = 0; j < NV; ++j) x[j] = j * THREADS + tid < n ? DT<T>::ld(in + j * THREADS + tid) : -INFINITY;
  const Settings set(a, r);
  const bool greedy = set.temperature == 0.f;
  const Slope c(set.temperature);
  bool bad = set.bad;
  float m = -INFINITY, low = INFINITY;
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    bad |= !(x[j] < INFINITY);
    x[j] = clean(x[j]);
    m = fmaxf(m, x[j]);
    if (x[j] > -INFINITY) low = fminf(low, x[j]);
  }
  if (bad) flag_status(a.status, DVI_DEV_NONFINITE);
  m = from_ord(__reduce_max_sync(0xffffffffu, ord(m)));
  low = from_ord(__reduce_min_sync(0xffffffffu, ord(low)));
  int at = NV;
#pragma unroll
  for (int j = NV - 1; j >= 0; --j)
    if (x[j] == m) at = j;
  at = __reduce_min_sync(0xffffffffu, at < NV ? at * THREADS + tid : 0x7fffffff);
  if (lane == 0) s.top[warp] = m, s.low[warp] = low, s.first[warp] = at;
  if (tid < 2) s.n_few[tid] = 0;
  if (tid < 2 * kFew) s.few[tid / kFew][tid % kFew] = make_ulonglong2(0, 0);
  __syncthreads();
  float top = -INFINITY;
  int hot = 0x7fffffff;
#pragma unroll
  for (int w = 0; w < THREADS / 32; ++w) {
    const float v = s.top[w];
    low = fminf(low, s.low[w]);
    if (v > top) top = v, hot = 0x7fffffff;
    if (v == top) hot = min(hot, s.first[w]);
  }
  if (greedy || top == -INFINITY) {
#pragma unroll
    for (int j = 0; j < NV; ++j)
      if (j * THREADS + tid < n) out[j * THREADS + tid] = top > -INFINITY && j * THREADS + tid == hot ? 1.f : 0.f;
    return;
  }
  Turns<THREADS> turns = {s};
  uint32_t o[NV];
#pragma unroll
  for (int j = 0; j < NV; ++j) o[j] = x[j] > -INFINITY ? ord(x[j]) : 0;
  unsigned long long mass[NV];
  const uint32_t least = ord(low);
  if (set.top_k) {
    Part all;
#pragma unroll
    for (int j = 0; j < NV; ++j) all.count += o[j] != 0;
    turns.template all<false>(all);
    if (all.count > static_cast<unsigned>(set.top_k)) cut_after<false, THREADS>(o, mass, set.top_k, all, least, ord(top), turns);
  }
  const Weigher weigher(top, c, nullptr);
  Part all;
#pragma unroll
  for (int j = 0; j < NV; j += 2) {
    unsigned high[2], rest[2];
    weigher.halves_by([&](unsigned i) { return weigher.entry(static_cast<int>(i), kPowersOf2.of); }, x[j], x[j + 1], high, rest);
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      mass[j + e] = o[j + e] ? Weigher::join(high[e], rest[e]) : 0;
      all.sum += mass[j + e];
      all.count += o[j + e] != 0;
    }
  }
  turns.template all<true>(all);
  unsigned long long kept = all.sum;
  if (set.top_p < 1.f)
    kept = cut_after<true, THREADS>(o, mass, share_of(set.top_p, kept), all, least, ord(top), turns);
  const Slope below = c.below();
  const float inv = 1.f / (__ull2float_rn(kept) * 0x1p-44f);
#pragma unroll
  for (int j = 0; j < NV; ++j)
    if (j * THREADS + tid < n) out[j * THREADS + tid] = o[j] ? weight(x[j], top, below) * inv : 0.f;
}

template <typename T, int NV, int THREADS, int CTAS_AN_SM>
cudaError_t launch_short(const TokenProbsArgs& a, cudaStream_t s) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(a.n_rows));
  cfg.blockDim = dim3(THREADS);
  cfg.stream = s;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, token_probs_short_kernel<T, NV, THREADS, CTAS_AN_SM>, a);
}

template <typename T>
cudaError_t launch_short(const TokenProbsArgs& a, cudaStream_t s) {
  if (a.vocab <= 8 * 128) return launch_short<T, 8, 128, 8>(a, s);
  static_assert(kShortRow == 8 * 256, "the longest");
  return launch_short<T, 8, 256, 4>(a, s);
}

}  // namespace

cudaError_t launch_probs_short(const TokenProbsArgs& a, int dtype, cudaStream_t s) {
  return dtype == DVI_BF16 ? launch_short<__nv_bfloat16>(a, s) : launch_short<float>(a, s);
}

}  // namespace dvi
