// Verification of drafted tokens from given uniform numbers.
//
// A cluster of CTAs takes a sequence: its first warps look at the drafts (a few
// words each), then all sum r = max(p - q, 0) over their parts of the row at
// which the drafts end, and the first CTA finds the token by descending to the
// part, the warp's share of it and the token at which the running sum passes u
// times the whole.  Which token that is does not depend on rounding but where u
// lies within 2^-40 of a border: p - q is exact as a pair of f32 numbers, its
// sums are pairs too (2^-48), and what is compared is in f64.
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

// hi + lo += a + b with |b| <= 2^-24 |a|.
__device__ __forceinline__ void add_pair(float& hi, float& lo, float a, float b) {
  const float s = __fadd_rn(hi, a), t = __fsub_rn(s, hi);
  lo = __fadd_rn(lo, __fadd_rn(__fadd_rn(__fsub_rn(hi, __fsub_rn(s, t)), __fsub_rn(a, t)), b));
  hi = s;
}

// A warp's sum of r over [lo, hi), on every lane.
__device__ double sum_range(const Residual& r, int lo, int hi, bool& bad) {
  const int lane = threadIdx.x & 31;
  float s = 0.f, e = 0.f;
  for (int i0 = lo; i0 < hi; i0 += kChunk) {
    float p[kFly], q[kFly];
#pragma unroll
    for (int j = 0; j < kFly; ++j) {
      const int i = i0 + 32 * j + lane;
      p[j] = i < hi ? r.p[i] : 0.f;
      q[j] = i < hi ? r.q_at(i) : 0.f;
    }
#pragma unroll
    for (int j = 0; j < kFly; ++j) {
      const float a = prob(p[j], bad), b = prob(q[j], bad);
      const float d = __fsub_rn(a, b), t = __fsub_rn(d, a);
      const float rest = __fsub_rn(__fsub_rn(a, __fsub_rn(d, t)), __fadd_rn(b, t));
      if (d > 0.f) add_pair(s, e, d, rest);
    }
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const float s2 = __shfl_xor_sync(0xffffffffu, s, o), e2 = __shfl_xor_sync(0xffffffffu, e, o);
    // (the same on both lanes: the larger first)
    const bool swap = s2 > s || (s2 == s && e2 > e);
    float hi = swap ? s2 : s, lo = swap ? e2 : e;
    add_pair(hi, lo, swap ? s : s2, swap ? e : e2);
    s = hi, e = lo;
  }
  return static_cast<double>(s) + static_cast<double>(e);
}

// Among n <= 32 * PER numbers >= 0 in order (a lane's lie together): the first up to which
// `base` and they sum to more than t, else the last that is above 0.  base: what is before it.
template <int PER>
__device__ int pick(const double (&v)[PER], double t, double& base) {
  const int lane = threadIdx.x & 31;
  double sum = 0.0;
#pragma unroll
  for (int j = 0; j < PER; ++j) sum += v[j];
  double incl = sum;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const double w = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += w;
  }
  double at = base + (incl - sum);
  int hit = -1, last = -1;
  double hit_at = 0.0, last_at = 0.0;
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    if (v[j] > 0.0) {
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

struct Small {
  double part[kMaxCtas * kWarps], sub[kWarps];
  int m, lo, hi, token;
  double base;
};

// The token within [0, V), where s.part holds the sums of the shares [i L, i L + L); called
// by all threads of a CTA.  -1 if there is none.
__device__ int find_token(const Residual& r, int V, int L, int shares, double u, Small& s, bool& bad) {
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  constexpr int kPer = kMaxCtas * kWarps / 32;
  double t = 0.0, base = 0.0;
  if (warp == 0) {
    double v[kPer], total = 0.0;
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      v[j] = lane * kPer + j < shares ? s.part[lane * kPer + j] : 0.0;
      total += v[j];
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
    t = u * total;
    const int share = pick(v, t, base);
    if (lane == 0) {
      s.lo = share < 0 ? -1 : share * L;
      s.hi = min(V, (share + 1) * L);
    }
  }
  __syncthreads();
  if (s.lo < 0) return -1;
  while (s.hi - s.lo > kChunk) {
    const int lo = s.lo, hi = s.hi, sub = (hi - lo + kThreads - 1) / kThreads * 32;
    const double v = sum_range(r, min(hi, lo + warp * sub), min(hi, lo + warp * sub + sub), bad);
    if (lane == 0) s.sub[warp] = v;
    __syncthreads();
    if (warp == 0) {
      const double one[1] = {lane < kWarps ? s.sub[lane] : 0.0};
      const int at = max(pick(one, t, base), 0);
      if (lane == 0) {
        s.lo = lo + at * sub;
        s.hi = min(hi, lo + at * sub + sub);
      }
    }
    __syncthreads();
  }
  if (warp == 0) {
    const int lo = s.lo, hi = s.hi;
    float p[kFly], q[kFly];
#pragma unroll
    for (int j = 0; j < kFly; ++j) {
      const int i = lo + lane * kFly + j;
      p[j] = i < hi ? r.p[i] : 0.f;
      q[j] = i < hi ? r.q_at(i) : 0.f;
    }
    double v[kFly];
#pragma unroll
    for (int j = 0; j < kFly; ++j)
      v[j] = fmax(static_cast<double>(prob(p[j], bad)) - static_cast<double>(prob(q[j], bad)), 0.0);
    const int at = pick(v, t, base);
    if (lane == 0) s.token = at < 0 ? -1 : lo + at;
  }
  __syncthreads();
  return s.token;
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
          rejected = !(static_cast<double>(a.u_accept[s0 + j]) * static_cast<double>(q) < static_cast<double>(p));
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
  int flags = 0;
  Residual r = {a.p + (row0 + m) * a.ld_p, nullptr, -1};
  if (m < K) {
    if (a.q) r.q = a.q + (s0 + m) * a.ld_q;
    r.hot = a.ids[s0 + m];
    if (r.hot < 0 || r.hot >= V) {
      flags = DVI_DEV_BAD_TOKEN;
      r.hot = -1;
    }
  }
  double v = 0.0;
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
    const float u_in = a.u_token[b];
    const double u = u_in >= 0.f ? static_cast<double>(u_in) : 0.0;
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

cudaError_t launch_verify_drafts(const VerifyArgs& a, cudaStream_t s) {
  int ctas = 1;
  while (ctas < kMaxCtas && static_cast<int64_t>(a.n_seqs) * ctas * 2 <= 608 && a.vocab / ctas > 2 * kThreads) ctas *= 2;
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
