// Verification of drafted tokens from given uniform numbers, one CTA a sequence.
#include "sample.cuh"

namespace dvi {
namespace {

constexpr int kThreads = 512;

// A probability as it counts: NaN, infinities and negative numbers are 0.
__device__ __forceinline__ float prob(float p, bool& bad) {
  if (!(fabsf(p) <= 3.402823466e38f)) {
    bad = true;
    return 0.f;
  }
  return fmaxf(p, 0.f);
}

__global__ void __launch_bounds__(kThreads) verify_drafts_kernel(VerifyArgs a) {
  __shared__ double part[kThreads / 32];
  __shared__ int s_m, s_bad, s_tok;
  griddep_wait();
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int b = blockIdx.x, V = a.vocab;
  const int per = a.start ? 0 : a.n_drafts / a.n_seqs;
  const int s0 = a.start ? min(max(a.start[b], 0), a.n_drafts) : b * per;
  const int s1 = a.start ? min(max(a.start[b + 1], s0), a.n_drafts) : s0 + per;
  const int K = min(s1 - s0, a.max_drafts);
  const int64_t row0 = static_cast<int64_t>(s0) + static_cast<int64_t>(b) * a.bonus;   // the target's
  const int width = a.max_drafts + a.bonus;
  int* out = a.out + static_cast<int64_t>(b) * width;
  int flags = 0;
  if (tid < 32) {
    int m = 0;
    for (; m < K; m += 32) {
      const int j = m + lane;
      bool rejected = j < K, bad = false;
      if (j < K) {
        const int id = a.ids[s0 + j];
        if (id >= 0 && id < V) {
          const float p = prob(a.p[(row0 + j) * a.ld_p + id], bad);
          const float q = a.q ? prob(a.q[(s0 + j) * a.ld_q + id], bad) : 1.f;
          if (bad) flags |= DVI_DEV_NONFINITE;
          rejected = !(static_cast<double>(a.u_accept[s0 + j]) * static_cast<double>(q) < static_cast<double>(p));
        }
      }
      const unsigned no = __ballot_sync(0xffffffffu, rejected);
      if (no) {
        m += __ffs(no) - 1;
        break;
      }
    }
    if (lane == 0) s_m = min(m, K), s_bad = 0, s_tok = -1;
  }
  __syncthreads();
  const int m = s_m;
  int token = -1;
  if (m < K || a.bonus) {
    const float* p = a.p + (row0 + m) * a.ld_p;
    const bool minus = m < K;
    const float* q = minus && a.q ? a.q + (s0 + m) * a.ld_q : nullptr;
    int hot = -1;
    if (minus) {
      hot = a.ids[s0 + m];
      if (hot < 0 || hot >= V) {
        flags |= DVI_DEV_BAD_TOKEN;
        hot = -1;
      }
    }
    double u = static_cast<double>(a.u_token[b]);
    if (!(u >= 0.0)) u = 0.0;
    const int seg = (V + kThreads - 1) / kThreads, lo = min(V, tid * seg), hi = min(V, lo + seg);
    bool bad = false;
    for (int pass = minus ? 0 : 1; pass < 2; ++pass) {
      auto value = [&](int i) {
        double v = static_cast<double>(prob(p[i], bad));
        if (pass == 0) v -= q ? static_cast<double>(prob(q[i], bad)) : (i == hot ? 1.0 : 0.0);
        return fmax(v, 0.0);
      };
      double sum = 0.0;
      for (int i = lo; i < hi; ++i) sum += value(i);
      double incl = sum;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const double w = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += w;
      }
      if (lane == 31) part[warp] = incl;
      __syncthreads();
      double at = incl - sum, total = 0.0;
      for (int w = 0; w < kThreads / 32; ++w) {
        if (w < warp) at += part[w];
        total += part[w];
      }
      if (total > 0.0) {
        const double t = u * total;
        int last = -1;
        for (int i = lo; i < hi; ++i) {
          const double v = value(i);
          if (v > 0.0) {
            last = i;
            at += v;
            if (at > t) break;
          }
        }
        // the first segment that reaches past t has the token; the last one with a number, if
        // rounding (or u = 1) leaves t past them all
        const bool hit = last >= 0 && at > t;
        const int key = hit ? last : last >= 0 ? V + (V - 1 - last) : 0x7fffffff;
        if (tid == 0) s_tok = 0x7fffffff;
        __syncthreads();
        if (key != 0x7fffffff) atomicMin(&s_tok, key);
        __syncthreads();
        token = s_tok < V ? s_tok : 2 * V - 1 - s_tok;
        break;
      }
      __syncthreads();
    }
    if (token < 0) flags |= DVI_DEV_NONFINITE;
    if (bad) flags |= DVI_DEV_NONFINITE;
  }
  if (flags) atomicOr(&s_bad, flags);
  for (int j = tid; j < width; j += kThreads) out[j] = j < m ? a.ids[s0 + j] : j == m && token >= 0 ? token : -1;
  if (tid == 0) {
    a.n_accepted[b] = m;
    a.n_committed[b] = m + (token >= 0 ? 1 : 0);
  }
  __syncthreads();
  if (tid == 0 && s_bad) flag_status(a.status, s_bad);
}

}  // namespace

cudaError_t launch_verify_drafts(const VerifyArgs& a, cudaStream_t s) {
  return launch_pdl(verify_drafts_kernel, dim3(a.n_seqs), dim3(kThreads), 0, s, a);
}

}  // namespace dvi
