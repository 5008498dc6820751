// Verification of drafted tokens from given uniform numbers.
//
// A cluster of CTAs takes a sequence: each looks at the drafts (a few words each),
// then all sum r = max(p - q, 0) over their shares of the row at which the drafts
// end, and the first CTA finds the token by descending to the share, the warp's
// part of it and the token at which the running sum passes u times the whole.
// Which token that is does not depend on the order of sums but where u lies within
// about 2^-44 of a border: p - q is exact as a pair of f32 numbers, its sums are
// pairs too, and from a warp's sum on they are whole numbers of 2^-61 of the whole
// (64-bit floating point is as slow here as a hundred of the other operations).
//
// Bound by memory where there is much of it: 128 sequences of 128001 tokens (two rows
// each, 131 MB) take 31 to 33 us, a dot product of them 27; 5 are the looks at the
// drafts and the search.  One sequence takes 6.7 us, a chain of five dependent loads.
// Copies by the bulk engine, 1 KB a warp and three ahead, took 48 us; the next numbers'
// loads under way in registers changed nothing.
#include <cooperative_groups.h>

#include "sample.cuh"

namespace dvi {
namespace {

namespace cg = cooperative_groups;

constexpr int kThreads = 512;
constexpr int kWarps = kThreads / 32;
constexpr int kMaxCtas = 8;        // of a sequence
constexpr int kFly = 8;            // numbers of each row that a thread has in flight
constexpr int kChunk = 32 * kFly;
constexpr int kLast = 2;           // numbers of a lane where a single warp finds the token

// A probability as it counts: NaN, infinities and negative numbers are 0.
__device__ __forceinline__ float prob(float p, bool& bad) {
  if (!(fabsf(p) <= 3.402823466e38f)) {
    bad = true;
    return 0.f;
  }
  return fmaxf(p, 0.f);
}

// The row that the token is taken from.
struct Residual {
  const float* p;
  const float* q;   // null: 1 at `hot`, 0 elsewhere
  int hot;
  __device__ __forceinline__ float q_at(int i) const { return q ? q[i] : i == hot ? 1.f : 0.f; }
};

// Two f32 numbers in one register pair: their sums take one instruction.
struct Two {
  unsigned long long v;
};
__device__ __forceinline__ Two two(float a, float b) {
  Two r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "f"(a), "f"(b));
  return r;
}
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
__device__ __forceinline__ Two operator-(Two a, Two b) {   // (the product with -1 is exact)
  Two r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(b.v), "l"(two(-1.f, -1.f).v), "l"(a.v));
  return r;
}

// (hi, lo) += a + b with |b| <= 2^-24 |a|.
template <typename F>
__device__ __forceinline__ void add_pair(F& hi, F& lo, F a, F b) {
  const F s = hi + a, t = s - hi;
  lo = lo + (((hi - (s - t)) + (a - t)) + b);
  hi = s;
}

// A warp's sum of r over [lo, hi) as a pair, on every lane.
__device__ float2 sum_range(const Residual& r, int lo, int hi, bool& bad) {
  const int lane = threadIdx.x & 31;
  Two s = two(0.f, 0.f), e = s, odd = s;
  for (int i0 = lo; i0 < hi; i0 += kChunk) {
    float p[kFly], q[kFly];
#pragma unroll
    for (int j = 0; j < kFly; ++j) {
      const int i = i0 + 32 * j + lane;
      p[j] = i < hi ? r.p[i] : 0.f;
      q[j] = i < hi ? r.q_at(i) : 0.f;
    }
#pragma unroll
    for (int j = 0; j < kFly; j += 2) {
      // 0 of finite numbers, NaN of others
      asm("fma.rn.f32x2 %0, %1, %2, %0;" : "+l"(odd.v) : "l"(two(p[j], p[j + 1]).v), "l"(two(0.f, 0.f).v));
      asm("fma.rn.f32x2 %0, %1, %2, %0;" : "+l"(odd.v) : "l"(two(q[j], q[j + 1]).v), "l"(two(0.f, 0.f).v));
      const float b0 = fmaxf(q[j], 0.f), b1 = fmaxf(q[j + 1], 0.f);
      const Two a = two(fmaxf(p[j], b0), fmaxf(p[j + 1], b1)), b = two(b0, b1);   // a >= b >= 0
      const Two d = a - b;
      add_pair(s, e, d, (a - d) - b);
    }
  }
  const float2 z = split(odd);
  if (__any_sync(0xffffffffu, !(z.x == 0.f && z.y == 0.f))) {
    // (again, and one by one: an infinity has come into the sums)
    bad = true;
    s = e = two(0.f, 0.f);
    for (int i = lo + lane; i < hi; i += 32) {
      const float b = prob(r.q_at(i), bad), a = fmaxf(prob(r.p[i], bad), b);
      const Two d = two(a, 0.f) - two(b, 0.f);
      add_pair(s, e, d, (two(a, 0.f) - d) - two(b, 0.f));
    }
  }
  float2 hi2 = split(s), lo2 = split(e);
  float h = hi2.x, l = lo2.x;
  add_pair(h, l, hi2.y, lo2.y);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const float h2 = __shfl_xor_sync(0xffffffffu, h, o), l2 = __shfl_xor_sync(0xffffffffu, l, o);
    // (the same on both lanes: the larger first)
    const bool swap = h2 > h || (h2 == h && l2 > l);
    float a = swap ? h2 : h, b = swap ? l2 : l;
    add_pair(a, b, swap ? h : h2, swap ? l : l2);
    h = a, l = b;
  }
  return make_float2(h, l);
}

// Pairs as whole numbers: times 2^k, k so that the largest is below 2^54 (and 128 of them below 2^61).
struct Scale {
  float a, b;   // 2^k = a b
  __device__ __forceinline__ unsigned long long of(float2 v) const {
    const long long w = __float2ll_rn(v.x * a * b) + __float2ll_rn(v.y * a * b);
    return w > 0 ? w : 0;
  }
};
__device__ __forceinline__ Scale scale_below(float most) {
  const int e = static_cast<int>(__float_as_uint(most) >> 23) - 126;   // most < 2^e
  const int k = 54 - e, half = k / 2;
  return {__int_as_float((half + 127) << 23), __int_as_float((k - half + 127) << 23)};
}

// Among n <= 32 * PER numbers in order (a lane's lie together): the first up to which
// `base` and they sum to more than t, else the last that is above 0.  base: what is before it.
template <int PER>
__device__ int pick(const unsigned long long (&v)[PER], unsigned long long t, unsigned long long& base) {
  const int lane = threadIdx.x & 31;
  unsigned long long sum = 0;
#pragma unroll
  for (int j = 0; j < PER; ++j) sum += v[j];
  unsigned long long incl = sum;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const unsigned long long w = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += w;
  }
  unsigned long long at = base + (incl - sum), hit_at = 0, last_at = 0;
  int hit = -1, last = -1;
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    if (v[j]) {
      last = j, last_at = at;
      if (hit < 0 && at + v[j] > t) hit = j, hit_at = at;
    }
    at += v[j];
  }
  const unsigned hits = __ballot_sync(0xffffffffu, hit >= 0), some = __ballot_sync(0xffffffffu, last >= 0);
  if (!some) return -1;
  const int from = hits ? __ffs(hits) - 1 : 31 - __clz(some);
  base = __shfl_sync(0xffffffffu, hits ? hit_at : last_at, from);
  return from * PER + __shfl_sync(0xffffffffu, hits ? hit : last, from);
}

// floor(u S) for u >= 0; S where u is 1 or more.
__device__ __forceinline__ unsigned long long share_of(float u, unsigned long long S) {
  if (!(u < 1.f)) return S;
  const uint32_t b = __float_as_uint(u);
  const int e = static_cast<int>(b >> 23);
  const unsigned long long f = e ? (b & 0x7fffffu) | 0x800000u : b & 0x7fffffu;
  const int shift = 150 - (e ? e : 1);                   // u = f 2^-shift, shift >= 24
  const unsigned long long lo = S * f, hi = __umul64hi(S, f);
  return shift < 64 ? (hi << (64 - shift)) + (lo >> shift) : shift < 128 ? hi >> (shift - 64) : 0;
}

struct Small {
  float2 part[kMaxCtas * kWarps], sub[kWarps];
  int m, lo, hi, token;
};

// The token within [0, V), where s.part holds the sums of the shares [i L, i L + L); called
// by all threads of a CTA.  -1 if there is none.
__device__ int find_token(const Residual& r, int V, int L, int shares, float u, Small& s, bool& bad) {
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  constexpr int kPer = kMaxCtas * kWarps / 32;
  unsigned long long t = 0, base = 0;
  Scale scale = {0.f, 0.f};
  if (warp == 0) {
    float2 part[kPer];
    float most = 0.f;
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      part[j] = lane * kPer + j < shares ? s.part[lane * kPer + j] : make_float2(0.f, 0.f);
      most = fmaxf(most, part[j].x);
    }
    most = warp_max(most);
    if (!(most <= 3.402823466e38f)) bad = true;   // the sum is past f32's range
    int share = -1;
    if (most > 0.f) {
      scale = scale_below(most);
      unsigned long long v[kPer], total = 0;
#pragma unroll
      for (int j = 0; j < kPer; ++j) total += v[j] = scale.of(part[j]);
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
      t = share_of(u, total);
      share = pick(v, t, base);
    }
    if (lane == 0) {
      s.lo = share < 0 ? -1 : share * L;
      s.hi = min(V, (share + 1) * L);
    }
  }
  __syncthreads();
  if (s.lo < 0) return -1;
  while (s.hi - s.lo > 32 * kLast) {
    const int lo = s.lo, hi = s.hi, sub = (hi - lo + kThreads - 1) / kThreads * 32;
    const float2 v = sum_range(r, min(hi, lo + warp * sub), min(hi, lo + warp * sub + sub), bad);
    if (lane == 0) s.sub[warp] = v;
    __syncthreads();
    if (warp == 0) {
      const float2 sub_sum = lane < kWarps ? s.sub[lane] : make_float2(0.f, 0.f);
      const unsigned long long one[1] = {scale.of(sub_sum)};
      int at = pick(one, t, base);
      // (parts below 2^-54 of the largest share alone: the first of them)
      const unsigned any = __ballot_sync(0xffffffffu, sub_sum.x > 0.f);
      if (at < 0) at = max(__ffs(any) - 1, 0);
      if (lane == 0) {
        s.lo = lo + at * sub;
        s.hi = min(hi, lo + at * sub + sub);
      }
    }
    __syncthreads();
  }
  if (warp == 0) {
    const int lo = s.lo, hi = s.hi;
    float p[kLast], q[kLast];
#pragma unroll
    for (int j = 0; j < kLast; ++j) {
      const int i = lo + lane * kLast + j;
      p[j] = i < hi ? r.p[i] : 0.f;
      q[j] = i < hi ? r.q_at(i) : 0.f;
    }
    unsigned long long v[kLast];
    bool above = false;
    int first = -1;
#pragma unroll
    for (int j = 0; j < kLast; ++j) {
      const float b = prob(q[j], bad), a = fmaxf(prob(p[j], bad), b), d = __fsub_rn(a, b);
      v[j] = scale.of(make_float2(d, __fsub_rn(__fsub_rn(a, d), b)));
      if (d > 0.f && first < 0) first = j, above = true;
    }
    int at = pick(v, t, base);
    // (numbers below 2^-54 of the largest share alone: the first of them)
    const unsigned any = __ballot_sync(0xffffffffu, above);
    if (at < 0 && any) at = (__ffs(any) - 1) * kLast + __shfl_sync(0xffffffffu, first, __ffs(any) - 1);
    if (lane == 0) s.token = at < 0 ? -1 : lo + at;
  }
  __syncthreads();
  return s.token;
}

// Whether u q < p, exactly.
__device__ __forceinline__ bool accepts(float u, float q, float p) {
  const float prod = __fmul_rn(u, q);
  if (fabsf(prod) < 0x1p-80f) return static_cast<double>(u) * static_cast<double>(q) < static_cast<double>(p);
  return prod < p || (prod == p && fmaf(u, q, -prod) < 0.f);
}

__global__ void __launch_bounds__(kThreads) verify_drafts_kernel(VerifyArgs a, int n_ctas, int L) {
  __shared__ Small s;
  cg::cluster_group cluster = cg::this_cluster();
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int rank = n_ctas > 1 ? static_cast<int>(cluster.block_rank()) : 0;
  const int b = blockIdx.x / n_ctas, V = a.vocab;
  if (n_ctas > 1) cluster_arrive_release();   // (waited for below: no CTA writes to one that is not there)
  griddep_wait();
  const int per = a.start ? 0 : a.n_drafts / a.n_seqs;
  const int s0 = a.start ? min(max(a.start[b], 0), a.n_drafts) : b * per;
  const int s1 = a.start ? min(max(a.start[b + 1], s0), a.n_drafts) : s0 + per;
  const int K = min(s1 - s0, a.max_drafts);
  const int64_t row0 = static_cast<int64_t>(s0) + static_cast<int64_t>(b) * a.bonus;   // the target's
  bool bad = false;
  const float u_in = a.u_token[b], u = u_in >= 0.f ? u_in : 0.f;
  if (warp == 0) {
    int m = 0;
    for (; m < K; m += 32) {
      const int j = m + lane;
      bool rejected = false;
      if (j < K) {
        const int id = a.ids[s0 + j];
        rejected = true;
        if (id >= 0 && id < V) {
          const float p = prob(a.p[(row0 + j) * a.ld_p + id], bad);
          const float q = a.q ? prob(a.q[(s0 + j) * a.ld_q + id], bad) : 1.f;
          rejected = !accepts(a.u_accept[s0 + j], q, p);
        }
      }
      const unsigned no = __ballot_sync(0xffffffffu, rejected);
      if (no) {
        m += __ffs(no) - 1;
        break;
      }
    }
    if (lane == 0) s.m = min(m, K);
  }
  __syncthreads();
  const int m = s.m;
  const bool some = m < K || a.bonus;
  int flags = a.start && (a.start[b] != s0 || a.start[b + 1] != s1) ? DVI_DEV_BAD_TOKEN : 0;
  Residual r = {a.p + (row0 + m) * a.ld_p, nullptr, -1};
  if (m < K) {
    if (a.q) r.q = a.q + (s0 + m) * a.ld_q;
    r.hot = a.ids[s0 + m];
    if (r.hot < 0 || r.hot >= V) {
      flags |= DVI_DEV_BAD_TOKEN;
      r.hot = -1;
    }
  }
  float2 v = make_float2(0.f, 0.f);
  const int share = rank * kWarps + warp;
  if (some) v = sum_range(r, min(V, share * L), min(V, share * L + L), bad);
  if (n_ctas > 1) {
    cluster_wait_acquire();
    if (lane == 0) *cluster.map_shared_rank(&s.part[share], 0) = v;
    cluster_arrive_release();
    if (rank) {
      if (bad) flag_status(a.status, DVI_DEV_NONFINITE);
      cluster_wait_acquire();
      return;
    }
    cluster_wait_acquire();
  } else {
    if (lane == 0) s.part[share] = v;
    __syncthreads();
  }
  int token = -1;
  if (some) {
    token = find_token(r, V, L, n_ctas * kWarps, u, s, bad);
    if (token < 0 && m < K) {
      // p is nowhere above q (by rounding: both sum to 1): a token of p, by this CTA alone
      r.q = nullptr, r.hot = -1;
      const int all = (V + kWarps - 1) / kWarps;
      v = sum_range(r, min(V, warp * all), min(V, warp * all + all), bad);
      if (lane == 0) s.part[warp] = v;
      __syncthreads();
      token = find_token(r, V, all, kWarps, u, s, bad);
    }
    if (token < 0) flags |= DVI_DEV_NONFINITE;
  }
  if (bad) flags |= DVI_DEV_NONFINITE;
  if (flags) flag_status(a.status, flags);
  const int width = a.max_drafts + a.bonus;
  int* out = a.out + static_cast<int64_t>(b) * width;
  for (int j = tid; j < width; j += kThreads) out[j] = j < m ? a.ids[s0 + j] : j == m && token >= 0 ? token : -1;
  if (tid == 0) {
    a.n_accepted[b] = m;
    a.n_committed[b] = m + (token >= 0 ? 1 : 0);
  }
}

}  // namespace

// As many CTAs a sequence as are resident at once (two an SM) and have something to do: 128 sequences of
// 128001 over 2 CTAs 30 us, over 4 37; 64 of 32000 over 4 10.7, over 8 14.2.
cudaError_t launch_verify_drafts(const VerifyArgs& a, cudaStream_t s) {
  int ctas = 1;
  while (ctas < kMaxCtas && static_cast<int64_t>(a.n_seqs) * ctas * 2 <= 304 && a.vocab / ctas > 2 * kThreads) ctas *= 2;
  const int shares = ctas * kWarps, L = ((a.vocab + shares - 1) / shares + 31) / 32 * 32;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(a.n_seqs) * ctas);
  cfg.blockDim = dim3(kThreads);
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
  return cudaLaunchKernelEx(&cfg, verify_drafts_kernel, a, ctas, L);
}

}  // namespace dvi
