// Probabilities of sampling from logits with tokens cut off: top-k, top-p.
//
// With tokens in the order of their logits (equal ones by index) and w =
// exp((x - max) / T), the kept tokens are a prefix of the order; it ends at the
// last token whose rank is below top_k and before which the sum of w is below
// top_p of the whole.  A row's slices lie in the shared memory of a cluster's CTAs.
//
// The last kept token is looked for in a histogram of the logits: of counts, or of w at the
// tokens' places in their bins by its tangent there, which gives a bin's sum to about 2^-15.
// The CTAs give each other their sums of 32 groups of 32 bins, then of the bins of the group in
// which the cut should be.  Then each sums w exactly, as whole numbers: of all tokens,
// of those before the bin, of those in it; these sums and the bin's tokens go to all.
// They show whether the bin is the right one (else it is its neighbour's turn) and,
// among its tokens, which is the last.  Every CTA comes to the same end, whatever the
// order of its atomics.  Where top_k leaves few tokens, all of these go to all instead,
// which is all that top_p needs, too.  Where the bin has too many tokens, a part of it is
// tried, where the cut would be if they lay evenly; where that has too many, too, the token's
// place in the order, as a number, is found 10 bits at a time (a row of 128001 with top_p 21 us;
// of equal logits, or of logits within 0.001, 160).
//
// What the CTAs give each other are stores that the receiver's barrier counts: no CTA
// waits for its own memory operations, as at a cluster's barrier (a block of 6 rows of
// 32000 with top_p: 14.3 us with the cluster's, 12.2 so).
//
// A few rows are bound by the chain of four exchanges and by code that is read for the
// first time (a third of the stalls): 6 rows of 32000 with top_p 11.2 us, 48 with top_k
// 50 12.7.  Many rows: of a CTA's time on a slice of 16000 tokens with top_p (50000 cycles) the
// exact sums take 14000 (instructions, and conflicts in the table of powers), the histogram 8000 (its
// atomics), the loads 6000, the stores 6000, and the exchanges between them the rest; with top_k 30000
// in all: 576 rows of 32000 108 and 65 us (a copy of them 23), 64 rows of 128001 with settings of their
// own 58 to 67 (17).  Further from a copy: flat rows, where a bin has too many tokens and the next try weighs
// all tokens again (64 rows of 128001 with T = 3 and top_p 0.9 104 us, with T = 1 71); top_k above 512, where
// all tokens down to the least of the threads' maxima are counted (576 rows of 32000, 900 likeliest, 123); short
// rows, which have as many barriers and as large a table as long ones (2000 of 4000 with top_p 77, without cuts 12.5).
#include "token_mass.cuh"

namespace dvi {
namespace {

constexpr int kThreads = 512;
constexpr int kWarps = kThreads / 32;
constexpr int kMaxCtas = kProbsCtas;
constexpr int kBins = 1024;                      // 32 groups of 32
constexpr int kBinBits = 10;
constexpr int kPer = kBins / kThreads;
constexpr int kRow = 128;                        // logits that a warp looks at together, four a thread
constexpr int kSteps = 1024;                     // places within a bin
constexpr float kBinsPerOctave = 40.f;           // of w
constexpr int kWide = 768;                       // from this bin on they are four times as wide: the last one has what
                                                 // is below 2^-44.6
constexpr float kFall = 0.69314718f / kBinsPerOctave;   // of w over a bin, by its tangent (a wide one: four times that)
// w at a bin's begin, less 1 for every step, where w falls by 1 over a step at the bin's middle; and what w is
// above its tangent, for tokens that lie evenly.
constexpr unsigned kTop = static_cast<unsigned>(kSteps * (1.f / kFall + 0.5f + kFall / 24.f) + 0.5f),
                   kTopWide = static_cast<unsigned>(kSteps * (0.25f / kFall + 0.5f + kFall / 6.f) + 0.5f);
static_assert(kMaxVocab / kMaxCtas * static_cast<unsigned long long>(kTop) < 1ull << 32, "a bin's sum");
constexpr int kList = 1024;                      // tokens of a bin that are sorted out by each CTA
constexpr int kListPer = kList / kThreads;
constexpr int kFew = 128;                        // tokens that are compared with each other, by four threads each
constexpr int kTries = 4;                        // parts of the histogram that are summed before the slow way is taken
constexpr int kIndexBits = 18;                   // kMaxVocab

__device__ __noinline__ unsigned long long mass_of(float x, float m, float c_hi, float c_lo, const float2* powers) {
  Slope c(1.f);
  c.hi = c_hi, c.lo = c_lo;
  const Weigher w(m, c, powers);
  unsigned high[2], rest[2];
  w.halves(x, x, high, rest);
  return Weigher::join(high[0], rest[0]);
}
// A thread's sum of masses: at most 64 halves of at most 2^22 each.
struct MassSum {
  unsigned high = 0, rest = 0;
  __device__ __forceinline__ void add(unsigned h, unsigned r) {
    high += h - Weigher::kBits;
    rest += r - Weigher::kBits;
  }
  // All of a pair; `of` says how many pairs there were.
  __device__ __forceinline__ void add(const unsigned (&h)[2], const unsigned (&r)[2]) {
    high += h[0] + h[1];
    rest += r[0] + r[1];
  }
  __device__ __forceinline__ void of(int pairs) {
    high -= 2 * pairs * Weigher::kBits;
    rest -= 2 * pairs * Weigher::kBits;
  }
  __device__ __forceinline__ unsigned long long value() const {
    return high * 4194304ull + static_cast<long long>(static_cast<int>(rest));
  }
};
static_assert(kMaxVocab / kMaxCtas <= 64 * kThreads, "64 logits a thread");

__device__ __forceinline__ unsigned long long warp_scan_u64(unsigned long long v) {   // inclusive
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const unsigned long long w = __shfl_up_sync(0xffffffffu, v, o);
    if (lane >= o) v += w;
  }
  return v;
}

// What a row needs beside its slice of logits.
struct Cuts {
  unsigned digit[3][kBins];                     // sums of the bins, by digits of 15 bits: no sum passes 32 bits,
                                                // and the atomics return nothing
  unsigned long long key[kList];                // the tokens of a bin, and their masses in the higher digits' place
  unsigned long long box[kList];                // as the CTAs send them, kList / n_ctas of each
  float2 powers[kPowers];
  __device__ __forceinline__ unsigned long long* mass() { return reinterpret_cast<unsigned long long*>(digit[1]); }
};
static_assert(2 * kBins * sizeof(unsigned) >= kList * sizeof(unsigned long long), "masses over the digits");

// What the CTAs of a cluster send each other, by rank, and what counts it.
struct Boxes {
  unsigned long long bar[6];                    // of: peers, groups, bins, sums, the list, kept
  float2 top[kMaxCtas];                         // maximum, least of the threads' maxima
  int2 first[kMaxCtas];                         // first token of the maximum, how many threads have a maximum
  float2 group[kMaxCtas][32];                   // sums of the groups of bins; .y of the first: how many tokens there are
  float2 bin[kMaxCtas][32];
  unsigned long long sum[2][4][kMaxCtas];       // (in turns) before the bin, in it, all; and how many are in it
  float2 kept[kMaxCtas];
};

struct Small {
  Boxes box;
  unsigned long long part[3][kWarps], least[kWarps], most[kWarps];
  float group[32];
  float red[kWarps], low[kWarps];
  int first[kWarps], some[kWarps];
  int n_list, n_kept, found;
  int vain;                                     // a warp has waited in vain
  int meetings;                                 // of the cluster, so far
  int lost;                                     // the one to which a CTA comes that has given up (none: -1)
  unsigned long long excl, cut, kept;
};

// One row (its slice in this CTA) and what is known of it.
struct RowState {
  const float* x;       // the slice, tokens first .. first + n - 1
  int first, n;         // (n: up to a multiple of kRow, with -inf behind the last token)
  int rank, n_ctas;
  float m;              // the row's maximum
  uint32_t top;         // ord(m)
  Slope c;
  int* status;
  Weigher mass;
  __device__ __forceinline__ unsigned long long place(float v, int i) const {
    return (static_cast<unsigned long long>(top - ord(v + 0.f)) << kIndexBits) | static_cast<unsigned>(first + i);
  }
  __device__ __forceinline__ float logit(unsigned long long place) const {
    return from_ord(top - static_cast<uint32_t>(place >> kIndexBits));
  }
  __device__ __forceinline__ unsigned long long mass_at(float v) const {
    return mass_of(v, m, c.hi, c.lo, mass.powers);
  }
  // The place in the histogram, down from the maximum: kSteps of them a bin, `scale` a unit
  // (rounded by adding 1.5 * 2^23).
  __device__ __forceinline__ int step(float v, float scale) const {
    const float t = __fmul_rn(__fsub_rn(m, v), scale);
    const float wide = fmaf(t, 0.25f, 0.75f * kWide * kSteps);
    return __float_as_int(__fadd_rn(fminf(fminf(t, wide), static_cast<float>(kBins * kSteps - 1)), 12582912.f)) & 0x1fffff;
  }
  // The same of two that are not below the last bins' end (of others: any number).
  __device__ __forceinline__ void steps(float v0, float v1, float scale, int (&to)[2]) const {
    const float2 t = split((two(m) - two(v0, v1)) * two(scale));
    const float2 wide = split(fma(two(t.x, t.y), two(0.25f), two(0.75f * kWide * kSteps)));
    const float2 at = split(two(fminf(t.x, wide.x), fminf(t.y, wide.y)) + two(12582912.f));
    to[0] = __float_as_int(at.x) - 0x4b400000;
    to[1] = __float_as_int(at.y) - 0x4b400000;
  }
  // (what lies before it, in bins of the first kind)
  static __device__ __forceinline__ float from(float bin) { return bin < kWide ? bin : kWide + 4.f * (bin - kWide); }
  __device__ __forceinline__ int bin(float v, float scale) const { return step(v, scale) / kSteps; }
};

// Eight bytes to the box of CTA r, counted by its k-th barrier.  (DVI_SENDS: whether they are, for a build that holds
// some back.)
#ifndef DVI_SENDS
#define DVI_SENDS(k, r) true
#endif
__device__ __forceinline__ void send(void* to, unsigned long long v, Boxes& box, int k, int r, int n_ctas) {
  if (n_ctas == 1) {
    *static_cast<unsigned long long*>(to) = v;
    return;
  }
  if (DVI_SENDS(k, r)) send_to(to, v, &box.bar[k], r);
}
// One thread says how much will come ...
__device__ __forceinline__ void expect(unsigned long long* bar, int bytes, int n_ctas) {
  if (n_ctas > 1) mbar_arrive_expect_tx(reinterpret_cast<uint64_t*>(bar), bytes);
}
// ... and all wait for it, a warp together.
__device__ __forceinline__ bool arrived(unsigned long long* bar, int turn, int n_ctas, int* status) {
  if (n_ctas > 1) return __all_sync(0xffffffffu, mbar_wait(reinterpret_cast<uint64_t*>(bar), turn & 1, status));
  __syncthreads();
  return true;
}

// A wait that runs out (a second: a CTA of the cluster has not sent what it should) costs the row, which gets zeros,
// in every CTA alike:
// - The CTA's first barrier behind a wait says whether a warp has waited in vain; one that has sends nothing more and
//   goes straight to that barrier.  (Between what it says and the next wait lies another barrier, so all see the same.)
// - If so, the CTA gives up: it leaves the number of the cluster's next meeting (its barrier) with all, and comes to
//   that meeting, which is its last.
// - The others find the number when they come there, if not before they have waited in vain themselves: it is
//   everybody's last.  So nobody leaves, or clears what others read, while a CTA might still send to it or read it,
//   and what a CTA goes on with has come whole from CTAs that had not given up.
// - A row that is right ends with a meeting, too, on whose way it is stored.
// (6 rows of 32000 with top_p 0.25 us of 12.6, half of it the last meeting; 576 with the 50 likeliest 1.3 of 64.7.)
__device__ __forceinline__ int now(const int& v) { return *static_cast<const volatile int*>(&v); }
__device__ __forceinline__ bool all_came(const Small& s) {
  __syncthreads();
  return now(s.vain) == 0;
}
__device__ __forceinline__ void in_vain(Small& s) {
  s.vain = 1;
  __syncthreads();
}
__device__ __forceinline__ bool meet(Small& s, int n_ctas) {   // (a barrier of the CTA lies between two of them)
  if (threadIdx.x == 0) ++s.meetings;
  cluster_barrier(n_ctas);
  return now(s.lost) != now(s.meetings);
}
// The last one, when nothing comes to this CTA or goes from it any more, and its end, when the row is stored.
__device__ __forceinline__ void arrive_at_last(int n_ctas) {
  if (n_ctas > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
}
// Zeros for a row that is lost; what was sent to this CTA before the last meeting (over: it is) has come when it ends.
__device__ __noinline__ void leave_zeros(float* probs, int64_t ld, int vocab, int n_ctas, int slice, Small& s, bool over) {
  if (!over && now(s.lost) != now(s.meetings)) {
    if (threadIdx.x < n_ctas) *cg::this_cluster().map_shared_rank(&s.lost, threadIdx.x) = now(s.meetings) + 1;
    __syncwarp();
    cluster_barrier(n_ctas);
  }
  __syncthreads();   // (behind what other threads have stored)
  const int first = static_cast<int>(cg::this_cluster().block_rank()) * slice;
  float* out = probs + blockIdx.x / n_ctas * ld;
  for (int i = first + threadIdx.x; i < min(first + slice, vocab); i += kThreads) out[i] = 0.f;
  for (const uint64_t t0 = global_ns(); global_ns() - t0 < 1000000;) {
  }
}

__device__ __forceinline__ void add_to_bin(Cuts& h, int bin, unsigned long long v) {
  const unsigned a = static_cast<unsigned>(v) & 0x7fffu, b = static_cast<unsigned>(v >> 15) & 0x7fffu,
                 c = static_cast<unsigned>(v >> 30);
  atomicAdd(&h.digit[0][bin], a);
  if (b) atomicAdd(&h.digit[1][bin], b);
  if (c) atomicAdd(&h.digit[2][bin], c);
}
__device__ __forceinline__ unsigned long long sum_of(unsigned a, unsigned b, unsigned c) {
  return a + (static_cast<unsigned long long>(b) << 15) + (static_cast<unsigned long long>(c) << 30);
}
__device__ __forceinline__ unsigned long long bin_sum(const Cuts& h, int bin) {
  return sum_of(h.digit[0][bin], h.digit[1][bin], h.digit[2][bin]);
}
__device__ __forceinline__ void clear_bins(Cuts& h) {
  for (int i = threadIdx.x; i < 3 * kBins; i += kThreads) (&h.digit[0][0])[i] = 0;
  __syncthreads();
}

// The first bin up to which the sums of CTAs r0 .. r1 - 1 (and `before`) reach target: its
// number (-1 if none does) and the sum before it.  Their bins are complete when it is called.
__device__ __noinline__ int find_bin(unsigned long long before, unsigned long long target, int r0, int r1, Cuts& h,
                                     Small& s, unsigned long long* excl) {
  cg::cluster_group cluster = cg::this_cluster();
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  static_assert(kPer == 2, "a pair of bins a thread");
  unsigned long long v[kPer] = {};
  for (int r = r0; r < r1; ++r) {
    uint2 d[3];
    for (int k = 0; k < 3; ++k) d[k] = reinterpret_cast<const uint2*>(cluster.map_shared_rank(h.digit[k], r))[tid];
    v[0] += sum_of(d[0].x, d[1].x, d[2].x);
    v[1] += sum_of(d[0].y, d[1].y, d[2].y);
  }
  const unsigned long long sum = v[0] + v[1], incl = warp_scan_u64(sum);
  if (lane == 31) s.part[0][warp] = incl;
  if (tid == 0) s.found = -1;
  __syncthreads();
  unsigned long long at = before + incl - sum;
  for (int w = 0; w < warp; ++w) at += s.part[0][w];
#pragma unroll
  for (int j = 0; j < kPer; ++j) {
    if (at < target && at + v[j] >= target) s.found = tid * kPer + j, s.excl = at;
    at += v[j];
  }
  __syncthreads();
  *excl = s.excl;
  return s.found;
}

// Of the n tokens in h.key (with h.mass()): the last kept one, where `before` is the sum before
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
      m[j] = i < n && MASS ? h.mass()[i] : 1;
      if (i < n) least = min(least, key[j]), most = max(most, key[j]);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      least = min(least, __shfl_xor_sync(0xffffffffu, least, o));
      most = max(most, __shfl_xor_sync(0xffffffffu, most, o));
    }
    if (lane == 0) s.least[warp] = least, s.most[warp] = most;
    if (tid == 0) s.n_kept = 0;
    __syncthreads();   // (the masses lie in the bins' place)
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
      if (MASS) h.mass()[at] = m[j];
    }
    __syncthreads();
    n = s.n_kept;
    __syncthreads();
  }
  {
    const int i = tid >> 2;
    const unsigned long long p = i < n ? h.key[i] : 0, v = i < n && MASS ? h.mass()[i] : 1;
    unsigned long long sum = 0;
    for (int j = tid & 3; j < n; j += 4)
      if (h.key[j] < p) sum += MASS ? h.mass()[j] : 1;
    sum += __shfl_xor_sync(0xffffffffu, sum, 1);
    sum += __shfl_xor_sync(0xffffffffu, sum, 2) + before;
    if ((tid & 3) == 0 && i < n && sum < target && sum + v >= target) s.cut = p, s.kept = sum + v;
  }
  __syncthreads();
  *kept = s.kept;
  return s.cut;
}

// First of the lanes up to which the numbers reach target (the last that is above 0, where rounding leaves
// it past all), and the sum before it.
__device__ __forceinline__ int first_reaching(float v, float target, float* before) {
  const int lane = threadIdx.x & 31;
  float incl = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const float w = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += w;
  }
  incl += *before;
  const unsigned at = __ballot_sync(0xffffffffu, v > 0.f && incl >= target), some = __ballot_sync(0xffffffffu, v > 0.f);
  if (!some) return -1;
  const int l = at ? __ffs(at) - 1 : 31 - __clz(some);
  *before = __shfl_sync(0xffffffffu, incl - v, l);
  return l;
}

// The last kept token among those up to `upto`: before it the counts sum to less than top_k (and then
// the masses to less than top_p of what top_k leaves: *done; else that is still to do), or (MASS) the
// masses to less than top_p of all.  Returns the tokens up to it.  *kept: the sum of their masses, where
// it is known (*done, or MASS).  Tokens below `low` are known to be cut (or, MASS, to be 0).  Where a wait
// has run out, here or elsewhere: a lost row.
//
// by_maxima (counts): the histogram has the largest logit of each thread alone (`mine`), which are at
// least top_k: the tokens that are not behind the bin in which the top_k-th of these lies are few more than
// top_k, and all are listed.  Where they do not fit, returns with *fits = false: then all tokens have to be
// counted.
template <bool MASS>
__device__ Upto last_kept(const RowState& row, int top_k, float top_p, Upto upto, float scale, float low, int (&turn)[3],
                          Cuts& h, Small& s, unsigned long long* kept, bool* done,
                          bool by_maxima = false, float mine = 0.f, bool* fits = nullptr) {
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, n_ctas = row.n_ctas, rank = row.rank;
  const float4* x4 = reinterpret_cast<const float4*>(row.x);
  const int n4 = row.n / 4;
  const bool all_of_them = upto.x == -INFINITY;
  Boxes& box = s.box;
  if (tid == 0) expect(&box.bar[1], n_ctas * 32 * 8, n_ctas);
  for (int i = tid; i < kBins; i += kThreads) h.digit[0][i] = 0;
  if (!all_came(s)) return Upto::lost_row();
  int some = 0;
  if (!MASS && by_maxima) {
    some = mine >= low && mine > -INFINITY;
    if (some) atomicAdd(&h.digit[0][row.bin(mine, scale)], 1u);
  }
  for (int g = !MASS && by_maxima ? n4 : tid; g < n4; g += kThreads) {
    const float4 q = x4[g];
    float v[4] = {q.x, q.y, q.z, q.w};
    if (MASS && !all_of_them) {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (!upto.has(v[e], 4 * g + e)) v[e] = -INFINITY;
    }
    const float top = fmaxf(fmaxf(v[0], v[1]), fmaxf(v[2], v[3]));
    if (!__any_sync(0xffffffffu, top >= low && top > -INFINITY)) continue;
#pragma unroll
    for (int e = 0; e < 4; e += 2) {
      int step[2];
      if (MASS)
        row.steps(v[e], v[e + 1], scale, step);   // (low is near the bins' end)
      else
        step[0] = row.step(v[e], scale), step[1] = row.step(v[e + 1], scale);
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const bool in = v[e + k] >= low && (MASS || v[e + k] > -INFINITY);   // (MASS: low is a number)
        if (!MASS) some += in;
        const int bin = step[k] / kSteps;
        if (in && step[k] < (kBins - 1) * kSteps)
          atomicAdd(&h.digit[0][bin], MASS ? (bin < kWide ? kTop : kTopWide) - static_cast<unsigned>(step[k] % kSteps) : 1u);
      }
    }
  }
  if (!MASS) {
    some = __reduce_add_sync(0xffffffffu, some);
    if (lane == 0) s.some[warp] = some;
  }
  __syncthreads();
  // The groups' sums to all.  Of masses: a bin's tokens have been added up as what w is at their places, in units
  // of its fall over a step, by the tangent at the bin's middle.
  auto bin_value = [&](int b) {
    const float sum = static_cast<float>(h.digit[0][b]);
    if (!MASS) return sum;
    return exp2f(0.5f * (row.from(b) + row.from(b + 1)) * (-1.f / kBinsPerOctave)) * sum *
           (b < kWide ? kFall / kSteps : 4.f * kFall / kSteps);
  };
#pragma unroll
  for (int j = 0; j < 32 / kWarps; ++j) {
    const int g = warp * (32 / kWarps) + j;
    const float v = warp_sum(bin_value(32 * g + lane));
    if (lane == 0) s.group[g] = v;
  }
  __syncthreads();
  if (warp < n_ctas) {   // (a warp for each)
    const int here = MASS ? 0 : __reduce_add_sync(0xffffffffu, lane < kWarps ? s.some[lane] : 0);
    send(&box.group[rank][lane], bits_of(s.group[lane], static_cast<float>(here)), box, 1, warp, n_ctas);
  }
  if (!arrived(&box.bar[1], turn[0] & 1, n_ctas, row.status)) {
    in_vain(s);
    return Upto::lost_row();
  }
  ++turn[0];
  float v = 0.f, tokens = 0.f;
#pragma unroll
  for (int r = 0; r < kMaxCtas; ++r) {
    const float2 p = r < n_ctas ? box.group[r][lane] : make_float2(0.f, 0.f);
    v += p.x;
    tokens += p.y;
  }
  if (!MASS && tokens < top_k) {              // (fewer tokens than top_k)
    // (all have read the sums before the next are sent)
    if (!all_came(s) || !meet(s, n_ctas)) return Upto::lost_row();
    return upto;
  }
  const float all_bins = warp_sum(v), about = MASS ? top_p * all_bins : static_cast<float>(top_k);
  float before_it = 0.f;
  const int group = all_bins >= about ? first_reaching(v, about, &before_it) : -1;
  int bin = -1, n = kList + 1;
  bool wide = false;   // (counts) all tokens up to the bin's are listed
  unsigned long long before = 0, target = top_k;
  const int cap = kList / n_ctas;
  if (group >= 0) {
    // the bins of the group in which the cut should be, to all
    if (tid == 0) expect(&box.bar[2], n_ctas * 32 * 8, n_ctas);
    if (warp < n_ctas)
      send(&box.bin[rank][lane], bits_of(bin_value(32 * group + lane), 0.f), box, 2, warp, n_ctas);
    if (!arrived(&box.bar[2], turn[1] & 1, n_ctas, row.status)) {
      in_vain(s);
      return Upto::lost_row();
    }
    ++turn[1];
    v = 0.f;
#pragma unroll
    for (int r = 0; r < kMaxCtas; ++r) v += r < n_ctas ? box.bin[r][lane].x : 0.f;
    bin = first_reaching(v, about, &before_it);
    if (bin >= 0) bin += 32 * group;
    before = static_cast<unsigned long long>(before_it);   // (of counts, which are exact)
    wide = !MASS && (by_maxima || before_it + __shfl_sync(0xffffffffu, v, bin & 31) <= kList);
  }
  int lo = bin * kSteps, hi = lo + kSteps;   // the part of the histogram that is looked at
  for (int tries = 0; lo >= 0 && hi <= (kBins - 1) * kSteps && tries < kTries; ++tries) {
    // Sums of the tokens before the part, in it and of all, and its tokens, to all.  Logits past `above`
    // are before it, below `under` behind it, by more than what rounding may do.
    const float width = kSteps / scale;
    const float above_it = row.m - row.from(lo * (1.f / kSteps) - 0.25f) * width,
                under_it = row.m - row.from(hi * (1.f / kSteps) + 0.25f) * width;
    const float above = above_it + 0x1p-21f * fmaxf(fabsf(row.m), fabsf(above_it)),
                under = under_it - 0x1p-21f * fmaxf(fabsf(row.m), fabsf(under_it));
    if (tid == 0) {
      expect(&box.bar[3], n_ctas * 4 * 8, n_ctas);
      s.n_list = 0;
    }
    if (!all_came(s)) return Upto::lost_row();
    MassSum ahead, within, all;
    int pairs = 0;
#pragma unroll 1
    for (int g = tid; g < n4; g += kThreads) {
      const float4 q = x4[g];
      float v[4] = {q.x, q.y, q.z, q.w};
      if (MASS && !all_of_them) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (!upto.has(v[e], 4 * g + e)) v[e] = -INFINITY;
      }
      const float top = fmaxf(fmaxf(v[0], v[1]), fmaxf(v[2], v[3]));
      const bool some = __any_sync(0xffffffffu, top >= under);
      if (MASS ? !__any_sync(0xffffffffu, top >= low) : !some) continue;
      pairs += 2;
#pragma unroll
      for (int k = 0; k < 4; k += 2) {
        unsigned high[2], rest[2];
        if (MASS) {
          row.mass.halves(v[k], v[k + 1], high, rest);
          all.add(high, rest);
          if (!some) continue;
        }
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          // (a token of the part is not below `low`, but all are where low is -inf)
          const float x = v[k + e];
          const bool past = x > above && !wide;
          if (MASS && past) ahead.add(high[e], rest[e]);
          if (past || !(x >= under && x > -INFINITY)) continue;
          const int step = row.step(x, scale);
          if (MASS && step < lo) ahead.add(high[e], rest[e]);
          if (step >= hi || (step < lo && !wide)) continue;
          if (MASS) within.add(high[e], rest[e]);
          const int to = atomicAdd(&s.n_list, 1);
          if (to >= cap) continue;
          const unsigned long long p = row.place(x, 4 * g + k + e);
#pragma unroll 1
          for (int r = 0; r < n_ctas; ++r) send(&h.box[rank * cap + to], p, box, 4, r, n_ctas);
        }
      }
    }
    all.of(pairs);
    unsigned long long sum[3] = {ahead.value(), within.value(), all.value()};
    if (MASS) {
#pragma unroll
      for (int k = 0; k < 3; ++k) {
        sum[k] = warp_sum_u64(sum[k]);
        if (lane == 0) s.part[k][warp] = sum[k];
      }
    }
    __syncthreads();
    if (warp < 4) {
      unsigned long long v = s.n_list;
      if (warp < 3) v = MASS ? warp_sum_u64(lane < kWarps ? s.part[warp][lane] : 0) : 0;
      if (lane < n_ctas) send(&box.sum[turn[2] & 1][warp][rank], v, box, 3, lane, n_ctas);
    }
    if (!arrived(&box.bar[3], turn[2] & 1, n_ctas, row.status)) {
      in_vain(s);
      return Upto::lost_row();
    }
    // (a lane a CTA)
    const int there = lane < n_ctas ? static_cast<int>(box.sum[turn[2] & 1][3][lane]) : 0;
    const int sent = __reduce_add_sync(0xffffffffu, min(there, cap));
    const int most = __reduce_max_sync(0xffffffffu, there);
    n = most > cap ? kList + 1 : sent;
    if (tid == 0) expect(&box.bar[4], sent * 8, n_ctas);
    bool here = MASS || !wide || n <= kList;   // (else the bin's tokens alone)
    if (!MASS && by_maxima) *fits = here;
    wide = wide && here;
    if (MASS) {
      unsigned long long in_it = 0, all = 0;
      before = 0;
#pragma unroll
      for (int r = 0; r < kMaxCtas; ++r) {
        if (r >= n_ctas) continue;
        const auto& sums = box.sum[turn[2] & 1];
        before += sums[0][r];
        in_it += sums[1][r];
        all += sums[2][r];
      }
      target = share_of(top_p, all);
      here = before < target && before + in_it >= target;
      const int span = hi - lo;
      if (!here) {
        lo += before >= target ? -span : span;
        hi = lo + span;
      } else if (n > kList && span > 1) {
        // as much of it as should have half of a list, where the cut would be if its tokens lay evenly
        const int part = max(1, span * (kList / 2) / (most * n_ctas));
        lo += min(max(static_cast<int>(__ull2float_rn(target - before) / __ull2float_rn(in_it) * span) - part / 2, 0),
                  span - part);
        hi = lo + part;
        here = false;
      }
    }
    if (!arrived(&box.bar[4], turn[2] & 1, n_ctas, row.status)) {
      in_vain(s);
      return Upto::lost_row();
    }
    ++turn[2];
    if (here) break;
    if (!MASS && by_maxima) return upto;
    n = kList + 1;
    // (all have what was sent before more is)
    if (!all_came(s)) return Upto::lost_row();
    if (!meet(s, n_ctas)) return Upto::lost_row();
  }
  unsigned long long cut;
  if (n <= kList) {
    // the warps share the CTAs' lists
    const int there = lane < n_ctas ? static_cast<int>(box.sum[(turn[2] & 1) ^ 1][3][lane]) : 0;
    const int per = kWarps / n_ctas, from = warp / per;
    const int before_them = __reduce_add_sync(0xffffffffu, lane < from ? there : 0);
    const int m = __shfl_sync(0xffffffffu, there, from);
    for (int i = warp % per * 32 + lane; i < m; i += per * 32) {
      const unsigned long long p = h.box[from * cap + i];
      h.key[before_them + i] = p;
      if (MASS) h.mass()[before_them + i] = row.mass_at(row.logit(p));
    }
    if (tid == 0) s.n_kept = 0;
    if (!all_came(s)) return Upto::lost_row();
    cut = last_of_list<MASS>(n, wide ? 0 : before, target, rank, h, s, kept);
    if (wide) {
      // the tokens that are left, and of these the last one of top_p
      __syncthreads();
      if (tid == 0) s.n_kept = 0;
      __syncthreads();
      unsigned long long all = 0;
      for (int i = warp % per * 32 + lane; i < m; i += per * 32) {
        const unsigned long long p = h.box[from * cap + i];
        if (p > cut) continue;
        const int to = atomicAdd(&s.n_kept, 1);
        h.key[to] = p;
        all += h.mass()[to] = row.mass_at(row.logit(p));
      }
      all = warp_sum_u64(all);
      if (lane == 0) s.part[0][warp] = all;
      __syncthreads();
      all = warp_sum_u64(lane < kWarps ? s.part[0][lane] : 0);
      *kept = all;
      *done = true;
      if (top_p < 1.f) {
        const int left = s.n_kept;
        __syncthreads();
        cut = last_of_list<true>(left, 0, share_of(top_p, all), rank, h, s, kept);
      }
    }
  } else {
    cg::cluster_group cluster = cg::this_cluster();
    if (!all_came(s)) return Upto::lost_row();
    if (MASS) {
      // (the sum of all, where no bin was looked at)
      unsigned long long all = 0;
      for (int i = tid; i < row.n; i += kThreads)
        if (row.x[i] >= low && upto.has(row.x[i], i)) all += row.mass_at(row.x[i]);
      all = warp_sum_u64(all);
      __syncthreads();
      if (lane == 0) s.part[1][warp] = all;
      if (!meet(s, n_ctas)) return Upto::lost_row();
      all = 0;
      for (int r = 0; r < n_ctas; ++r)
        for (int w = 0; w < kWarps; ++w) all += cluster.map_shared_rank(&s, r)->part[1][w];
      target = share_of(top_p, all);
    }
    before = cut = 0;
    for (int shift = 32 + kIndexBits - kBinBits;; shift = shift > kBinBits ? shift - kBinBits : 0) {
      __syncthreads();
      clear_bins(h);
      for (int i = tid; i < row.n; i += kThreads) {
        const float x = row.x[i];
        if (!(x > -INFINITY) || !upto.has(x, i)) continue;
        const unsigned long long p = row.place(x, i);
        if (p < cut || ((p - cut) >> shift) >= kBins) continue;
        add_to_bin(h, static_cast<int>((p - cut) >> shift), MASS ? row.mass_at(x) : 1ull);
      }
      if (!meet(s, n_ctas)) return Upto::lost_row();
      const int b = find_bin(before, target, 0, n_ctas, h, s, &before);   // (found: the whole reaches target)
      cut += static_cast<unsigned long long>(b) << shift;
      if (shift == 0) {
        // one token a bin
        *kept = before;
        for (int r = 0; r < n_ctas; ++r) *kept += bin_sum(*cluster.map_shared_rank(&h, r), b);
      }
      if (!meet(s, n_ctas)) return Upto::lost_row();   // before the bins are cleared
      if (shift == 0) break;
    }
  }
  return {row.logit(cut), static_cast<int>(cut & ((1u << kIndexBits) - 1)) - row.first};
}

// How a row's logits and probabilities are taken: one by one, 16 bytes at a time, or so but for the ends of rows that
// begin anywhere (64 rows of 128001, the 50 likeliest, 33.5 us, one by one 38.5; 576 of 32000 with top_p as if they
// began anywhere 106.7, else 104.2).
enum How { kSingle, kWhole, kRagged };

// Ragged: a slice begins at the 16 bytes that its first logit lies in, `skip` logits earlier, where the probabilities'
// 16 bytes begin, too.
template <typename T>
bool rows_alike(const TokenProbsArgs& a) {
  return (reinterpret_cast<uintptr_t>(a.x) / sizeof(T) - reinterpret_cast<uintptr_t>(a.out) / 4) % 4 == 0 &&
         (a.n_rows == 1 || (a.ld - a.ld_out) % 4 == 0);
}
// The logits from i on that are within [from, to), -inf for others.
template <How HOW, typename T>
__device__ __forceinline__ void load_within(const T* p, int i, int from, int to, float* v) {
  constexpr int K = 16 / sizeof(T);
  if (HOW == kWhole ? i < to : i >= from && i + K <= to) {
    load16(p + i, v);
  } else {
#pragma unroll
    for (int e = 0; e < K; ++e) v[e] = HOW == kRagged && i + e >= from && i + e < to ? DT<T>::ld(p + i + e) : -INFINITY;
  }
}
template <How HOW>
__device__ __forceinline__ void store_within(float* p, int i, int from, int to, float4 v) {
  if (HOW == kWhole ? i < to : i >= from && i + 4 <= to) {
    *reinterpret_cast<float4*>(p + i) = v;
  } else if (HOW == kRagged) {
    if (i >= from && i < to) p[i] = v.x;
    if (i + 1 >= from && i + 1 < to) p[i + 1] = v.y;
    if (i + 2 >= from && i + 2 < to) p[i + 2] = v.z;
    if (i + 3 >= from && i + 3 < to) p[i + 3] = v.w;
  }
}

template <typename T, How HOW>
__global__ void __launch_bounds__(kThreads, 2) token_probs_cut_kernel(TokenProbsArgs a, int n_ctas, int slice) {
  extern __shared__ __align__(16) unsigned char dynamic[];
  __shared__ Small s;
  Cuts& h = *reinterpret_cast<Cuts*>(dynamic);
  float* x = reinterpret_cast<float*>(dynamic + sizeof(Cuts));
  float4* x4 = reinterpret_cast<float4*>(x);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int rank = n_ctas > 1 ? static_cast<int>(cg::this_cluster().block_rank()) : 0;
  const int r = blockIdx.x / n_ctas;
  int first = min(rank * slice, a.vocab), n = min(slice, a.vocab - first);
  Boxes& box = s.box;
  if (tid < 6) {
    mbar_init(reinterpret_cast<uint64_t*>(&box.bar[tid]), 1);
    mbar_fence_init();
    if (tid == 0) expect(&box.bar[0], n_ctas * 16, n_ctas);
    if (tid == 5) expect(&box.bar[5], n_ctas * 8, n_ctas);
    if (tid == 0) s.meetings = 0, s.lost = -1, s.vain = 0;
  }
  if (n_ctas > 1) cluster_arrive_release();              // (waited for before anything is sent)
  griddep_wait();
  const T* in = static_cast<const T*>(a.x) + r * a.ld + first;
  float* out = a.out + r * a.ld_out + first;
  constexpr bool WIDE = HOW != kSingle;
  const int skip = HOW == kRagged && n ? reinterpret_cast<uintptr_t>(in) / sizeof(T) % (16 / sizeof(T)) : 0;
  in -= skip, out -= skip, first -= skip, n += skip;
  const int n4 = (n + kRow - 1) / kRow * (kRow / 4);

  static_assert(kPowers == 2 * kThreads, "two each");
  h.powers[tid] = kPowersOf2.of[tid];
  h.powers[tid + kThreads] = kPowersOf2.of[tid + kThreads];
  float own = -INFINITY;
  bool odd = false;   // NaN or +inf among them
  constexpr int kFly = WIDE ? 16 : 32;   // logits of a thread on their way
  constexpr int kTogether = WIDE ? 16 / sizeof(T) : 1;
  if constexpr (WIDE) {
    for (int g0 = 0; g0 * kTogether < n; g0 += kFly / kTogether * kThreads) {
      float v[kFly];
#pragma unroll
      for (int j = 0; j < kFly; j += kTogether) {
        load_within<HOW>(in, (g0 + j / kTogether * kThreads + tid) * kTogether, skip, n, &v[j]);
      }
#pragma unroll
      for (int j = 0; j < kFly; j += kTogether) {
        const int i = (g0 + j / kTogether * kThreads + tid) * kTogether;
        if (i >= n) continue;
#pragma unroll
        for (int e = 0; e < kTogether; ++e) {
          own = fmaxf(own, v[j + e]);
          odd |= !(v[j + e] < INFINITY);
        }
#pragma unroll
        for (int e = 0; e < kTogether; e += 4)
          x4[(i + e) / 4] = make_float4(v[j + e], v[j + e + 1], v[j + e + 2], v[j + e + 3]);
      }
    }
  } else {
    int i0 = 0;
    for (; i0 + kFly * kThreads <= n; i0 += kFly * kThreads) {
      float v[kFly];
#pragma unroll
      for (int j = 0; j < kFly; ++j) v[j] = DT<T>::ld(in + i0 + j * kThreads + tid);
#pragma unroll
      for (int j = 0; j < kFly; ++j) {
        own = fmaxf(own, v[j]);
        odd |= !(v[j] < INFINITY);
        x[i0 + j * kThreads + tid] = v[j];
      }
    }
    if (i0 < n) {
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
        odd |= !(v[j] < INFINITY);
        if (i < n) x[i] = v[j];
      }
    }
  }
  if (const int i = (n + kTogether - 1) / kTogether * kTogether + tid; i < 4 * n4) x[i] = -INFINITY;
  const Settings set(a, r);
  const bool greedy = set.temperature == 0.f;
  const Slope c(set.temperature);
  // the tokens that the thread has loaded
  auto each = [&](auto f) {
    if (WIDE) {
#pragma unroll 1
      for (int g = tid; g * kTogether < n; g += kThreads)
#pragma unroll 1
        for (int i = g * kTogether; i < (g + 1) * kTogether; ++i) f(i);
    } else {
#pragma unroll 1
      for (int i = tid; i < n; i += kThreads) f(i);
    }
  };
  bool bad = set.bad;
  if (__syncthreads_or(odd)) {
    own = -INFINITY;
    each([&](int i) {
      bad |= !(x[i] < INFINITY);
      x[i] = clean(x[i]);
      own = fmaxf(own, x[i]);
    });
  }
  if (bad) flag_status(a.status, DVI_DEV_NONFINITE);
  {
    // the CTA's maximum and its first token, and the least of the threads' maxima, to all
    const float m = from_ord(__reduce_max_sync(0xffffffffu, ord(own)));
    const float low = from_ord(__reduce_min_sync(0xffffffffu, own > -INFINITY ? ord(own) : 0xff7fffffu));
    const unsigned some = __ballot_sync(0xffffffffu, own > -INFINITY);
    int at = 0x7fffffff;
    if (greedy) {
      if (m > -INFINITY && own == m)
        each([&](int i) {
          if (x[i] == m) at = min(at, first + i);
        });
      at = __reduce_min_sync(0xffffffffu, at);
    }
    if (lane == 0) s.red[warp] = m, s.low[warp] = low, s.first[warp] = at, s.some[warp] = __popc(some);
  }
  __syncthreads();
  if (n_ctas > 1) cluster_wait_acquire();
  if (warp == 0) {
    const bool is = lane < kWarps;
    const float w = is ? s.red[lane] : -INFINITY;
    const float m = from_ord(__reduce_max_sync(0xffffffffu, ord(w)));
    const float low = from_ord(__reduce_min_sync(0xffffffffu, is ? ord(s.low[lane]) : 0xff7fffffu));
    const int at = __reduce_min_sync(0xffffffffu, is && w == m ? s.first[lane] : 0x7fffffff);
    const int some = __reduce_add_sync(0xffffffffu, is ? s.some[lane] : 0);
    if (lane < n_ctas) {
      send(&box.top[rank], bits_of(m, low), box, 0, lane, n_ctas);
      send(&box.first[rank], (static_cast<unsigned long long>(some) << 32) | static_cast<unsigned>(at), box, 0,
           lane, n_ctas);
    }
  }
  int turn[3] = {0, 0, 0};
  const bool came = arrived(&box.bar[0], 0, n_ctas, a.status);
  const bool is = lane < n_ctas;
  const float2 of_cta = is ? box.top[lane] : make_float2(-INFINITY, 3.402823466e38f);
  const int2 first_of = is ? box.first[lane] : make_int2(0x7fffffff, 0);
  const float top = from_ord(__reduce_max_sync(0xffffffffu, ord(of_cta.x)));
  const RowState row = {x, first, 4 * n4, rank, n_ctas, top, ord(top + 0.f), c, a.status, Weigher(top, c, h.powers)};
  {
    const float2 e0 = row.mass.entry(tid, h.powers), e1 = row.mass.entry(tid + kThreads, h.powers);
    if (!came) s.vain = 1;
    if (!all_came(s)) return leave_zeros(a.out, a.ld_out, a.vocab, n_ctas, slice, s, false);
    h.powers[tid] = e0;
    h.powers[tid + kThreads] = e1;   // (read behind the next barrier)
  }
  auto nothing = [&](bool over) { leave_zeros(a.out, a.ld_out, a.vocab, n_ctas, slice, s, over); };
  auto last_wait = [&] {
    if (n_ctas == 1) return;
    cluster_wait_acquire();
    if (now(s.lost) == s.meetings + 1) nothing(true);
  };
  if (greedy || top == -INFINITY) {
    arrive_at_last(n_ctas);
    const int hot = __reduce_min_sync(0xffffffffu, of_cta.x == top ? first_of.x : 0x7fffffff);
    for (int i = skip + tid; i < n; i += kThreads) out[i] = top > -INFINITY && first + i == hot ? 1.f : 0.f;
    last_wait();
    return;
  }
  Upto upto = {-INFINITY, 0x7fffffff};
  unsigned long long kept = 0;
  bool done = false;
  if (set.top_k) {
    // Bins from the maximum down to the least of the threads' maxima, where there are top_k
    // of these (so many tokens are not below it); else as for the masses.
    const float low = from_ord(__reduce_min_sync(0xffffffffu, ord(of_cta.y)));
    const bool enough = set.top_k <= __reduce_add_sync(0xffffffffu, first_of.y);
    Upto cut;
    for (bool by_maxima = enough && set.top_k <= kList / 2, fits = false; !fits; by_maxima = false) {
      fits = true;
      cut = last_kept<false>(row, set.top_k, set.top_p, upto,
                             enough ? fminf(row.from(kBins - 2) * kSteps / (top - low), 1e30f)
                                    : c.hi * (kSteps * kBinsPerOctave),
                             enough ? low : -INFINITY, turn, h, s, &kept, &done, by_maxima, own, &fits);
      if (cut.lost()) return nothing(false);
    }
    upto = cut;
  }
  float inv;
  if (done) {
    inv = 1.f / (__ull2float_rn(kept) * 0x1p-44f);
  } else if (set.top_p < 1.f) {
    // (a mass is 0 below 2^-46)
    upto = last_kept<true>(row, 0, set.top_p, upto, c.hi * (kSteps * kBinsPerOctave), row.mass.low(), turn, h, s, &kept,
                           &done);
    if (upto.lost()) return nothing(false);
    inv = 1.f / (__ull2float_rn(kept) * 0x1p-44f);
  } else {
    const Slope below = c.below();
    float sum = 0.f;
    for (int g = tid; g < n4; g += kThreads) {
      const float4 q = x4[g];
      const float v[4] = {q.x, q.y, q.z, q.w};
      if (!__any_sync(0xffffffffu, fmaxf(fmaxf(v[0], v[1]), fmaxf(v[2], v[3])) >= upto.x)) continue;
#pragma unroll
      for (int e = 0; e < 4; ++e) sum += upto.has(v[e], 4 * g + e) ? weight(v[e], top, below) : 0.f;
    }
    sum = warp_sum(sum);
    if (lane == 0) s.red[warp] = sum;
    __syncthreads();
    if (warp == 0) {
      sum = warp_sum(lane < kWarps ? s.red[lane] : 0.f);
      if (lane < n_ctas) send(&box.kept[rank], bits_of(sum, 0.f), box, 5, lane, n_ctas);
    }
    if (!arrived(&box.bar[5], 0, n_ctas, a.status)) s.vain = 1;
    if (!all_came(s)) return nothing(false);
    sum = 0.f;
    for (int q = 0; q < n_ctas; ++q) sum += box.kept[q].x;
    inv = 1.f / sum;
  }
  arrive_at_last(n_ctas);
  const Slope below = c.below();
  auto prob = [&](float v, int i) { return upto.has(v, i) ? weight(v, top, below) * inv : 0.f; };
  // (most tokens are cut off, mostly whole warps of them)
  if (WIDE) {
    for (int g = tid; g < n4; g += kThreads) {
      const float4 q = x4[g];
      const int i = 4 * g;
      float4 p = make_float4(0.f, 0.f, 0.f, 0.f);
      if (__any_sync(0xffffffffu, fmaxf(fmaxf(q.x, q.y), fmaxf(q.z, q.w)) >= upto.x))
        p = make_float4(prob(q.x, i), prob(q.y, i + 1), prob(q.z, i + 2), prob(q.w, i + 3));
      store_within<HOW>(out, i, skip, n, p);
    }
  } else {
    for (int i0 = tid; i0 < 4 * n4; i0 += 4 * kThreads) {
      float v[4], m = -INFINITY;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        v[j] = i0 + j * kThreads < 4 * n4 ? x[i0 + j * kThreads] : -INFINITY;
        m = fmaxf(m, v[j]);
      }
      const bool some = __any_sync(0xffffffffu, m >= upto.x);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int i = i0 + j * kThreads;
        if (i < n) out[i] = some ? prob(v[j], i) : 0.f;
      }
    }
  }
  last_wait();
}

constexpr int kSlice = 16384;   // logits of a CTA where its row may have up to kMaxCtas: two CTAs an SM

// As few CTAs as hold a row in slices, and more while there are fewer than SMs (152) and the slices are
// worth it: 6 rows of 32000 with top_p over 8 CTAs 11.2 us, over 4 13.0, over 2 17.4; 48 rows over 4 18.0, over
// 2 20.4, over 8 (more than are resident) 25.8.
template <typename T, How HOW>
cudaError_t launch_cut(const TokenProbsArgs& a, cudaStream_t s) {
  static PerDevice per_device;
  per_device.once([&] {
    cudaFuncSetAttribute(token_probs_cut_kernel<T, HOW>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                         (kMaxVocab / kMaxCtas + 2 * kRow) * static_cast<int>(sizeof(float)) + static_cast<int>(sizeof(Cuts)));
  });
  int ctas = 1;
  while (ctas < kMaxCtas && (ctas * kSlice < a.vocab || (static_cast<int64_t>(a.n_rows) * ctas < 152 && a.vocab / ctas > 4096)))
    ctas *= 2;
  return launch_rows(token_probs_cut_kernel<T, HOW>, a, ctas, kThreads, sizeof(Cuts) + 2 * kRow * sizeof(float), sizeof(float), s);
}
template <typename T>
cudaError_t launch_cut(const TokenProbsArgs& a, cudaStream_t s) {
  if (rows_aligned<T>(a)) return launch_cut<T, kWhole>(a, s);
  return rows_alike<T>(a) ? launch_cut<T, kRagged>(a, s) : launch_cut<T, kSingle>(a, s);
}

}  // namespace

cudaError_t launch_probs_cut(const TokenProbsArgs& a, int dtype, cudaStream_t s) {
  return dtype == DVI_BF16 ? launch_cut<__nv_bfloat16>(a, s) : launch_cut<float>(a, s);
}

}  // namespace dvi
