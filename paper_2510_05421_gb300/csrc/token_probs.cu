// Probabilities of sampling from logits where nothing is cut off: softmax(x / T).
//
// The CTAs of a cluster hold a row between them in registers, so it is read once, and
// every warp gives (its maximum, its sum of exp2) to all of them once.
//
// Bound by memory and that exchange: 576 rows of 32000 f32 logits (147 MB) take 30 us
// (4.9 TB/s), of which the exchange is 5.5, a copy of them 23 us; of bf16 logits (110 MB), whose
// 16 bytes a lane are 32 bytes of probabilities in two stores, 31.  (Of the 64 registers a thread that
// leave room for four CTAs some 70 bytes are spilled.)  32
// logits a thread and four CTAs of 256 threads an SM: 16 a thread 34 us, 64 a thread 37,
// clusters that take row after row with the next one's loads under way 32, a row a CTA
// with the next one's bulk copy under way 35.
#include "token_probs.cuh"

namespace dvi {
namespace {

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

// Rows without cuts: NV logits a thread, in registers; 16 bytes at a time (WIDE) or one by one.  A warp
// takes w to its own maximum.
template <typename T, int NV, int THREADS, int CTAS_AN_SM, bool WIDE>
__global__ void __launch_bounds__(THREADS, CTAS_AN_SM)
    token_probs_kernel(TokenProbsArgs a, int n_ctas, int slice) {
  __shared__ float2 peer[kProbsCtas * THREADS / 32];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int rank = n_ctas > 1 ? static_cast<int>(cg::this_cluster().block_rank()) : 0;
  const int r = blockIdx.x / n_ctas;
  const int first = min(rank * slice, a.vocab), n = min(slice, a.vocab - first);
  // (that it is there: waited for before anything is written to it)
  if (n_ctas > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
  griddep_wait();
  const T* in = static_cast<const T*>(a.x) + r * a.ld + first;
  float* out = a.out + r * a.ld_out + first;
  constexpr int kTogether = WIDE ? 16 / sizeof(T) : 1;
  auto index = [&](int j) { return (j / kTogether * THREADS + tid) * kTogether + j % kTogether; };
  float v[NV];
  if constexpr (WIDE) {
#pragma unroll
    for (int j = 0; j < NV; j += kTogether) {
      const int i = index(j);
      if (i < n) {
        load16(in + i, &v[j]);
      } else {
#pragma unroll
        for (int e = 0; e < kTogether; ++e) v[j + e] = -INFINITY;
      }
    }
  } else {
#pragma unroll
    for (int j = 0; j < NV; ++j) v[j] = index(j) < n ? DT<T>::ld(in + index(j)) : -INFINITY;
  }
  const Settings set(a, r);
  const bool greedy = set.temperature == 0.f;
  const Slope c = Slope(set.temperature).below();
  bool bad = set.bad;
  float m = -INFINITY;
  bool odd = false;   // NaN or +inf among them
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    m = fmaxf(m, v[j]);
    odd |= !(v[j] < INFINITY);
  }
  if (__any_sync(0xffffffffu, odd)) {
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
  if (greedy) {
    int at = NV;
#pragma unroll
    for (int j = NV - 1; j >= 0; --j)
      if (v[j] == m) at = j;
    mine.y = __int_as_float(__reduce_min_sync(0xffffffffu, at < NV ? first + index(at) : 0x7fffffff));
  } else if (m > -INFINITY) {
    float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < NV; ++j) sum[j & 3] += v[j] = weight(v[j], m, c);
    mine.y = warp_sum((sum[0] + sum[1]) + (sum[2] + sum[3]));
  }
  if (bad) flag_status(a.status, DVI_DEV_NONFINITE);
  if (n_ctas > 1) {
    cluster_wait_acquire();
    if (lane < n_ctas) *cg::this_cluster().map_shared_rank(&peer[rank * (THREADS / 32) + warp], lane) = mine;
  } else if (lane == 0) {
    peer[warp] = mine;
  }
  cluster_barrier(n_ctas);
  float top, sum;
  int hot;
  join<THREADS / 32>(peer, n_ctas, greedy, c, &top, &sum, &hot);
  float scale = 0.f;
  if (!greedy && m > -INFINITY) {
    scale = weight(m, top, c) / sum;
  } else {
#pragma unroll
    for (int j = 0; j < NV; ++j) v[j] = 0.f;
  }
  if constexpr (WIDE) {
#pragma unroll
    for (int j = 0; j < NV; j += kTogether) {
      const int i = index(j);
      if (i >= n) continue;
#pragma unroll
      for (int e = 0; e < kTogether; e += 4)
        *reinterpret_cast<float4*>(out + i + e) = make_float4(v[j + e] * scale, v[j + e + 1] * scale,
                                                              v[j + e + 2] * scale, v[j + e + 3] * scale);
    }
  } else {
#pragma unroll
    for (int j = 0; j < NV; ++j)
      if (index(j) < n) out[index(j)] = v[j] * scale;
  }
  if (greedy && top > -INFINITY && hot >= first && hot < first + n) {
    __syncthreads();   // (behind the 0 that another thread has stored there)
    if (tid == 0) out[hot - first] = 1.f;
  }
}

template <typename T, bool WIDE, int NV, int THREADS, int CTAS_AN_SM>
cudaError_t launch_plain(const TokenProbsArgs& a, cudaStream_t s) {
  int ctas = 1;
  while (ctas * NV * THREADS < a.vocab) ctas *= 2;
  return launch_rows(token_probs_kernel<T, NV, THREADS, CTAS_AN_SM, WIDE>, a, ctas, THREADS, 0, 0, s);
}

// One CTA for rows of up to 8192 logits, of no more threads and logits a thread than the row needs (4096
// rows of 1024: 128 threads with 8 each 9 us, 256 with 32 33; of 4000: 256 with 16 22, 512 with 16 40); then
// as few as hold a row.
template <typename T, bool WIDE>
cudaError_t launch_plain(const TokenProbsArgs& a, cudaStream_t s) {
  if (a.vocab <= 8 * 128) return launch_plain<T, WIDE, 8, 128, 12>(a, s);
  if (a.vocab <= 16 * 128) return launch_plain<T, WIDE, 16, 128, 12>(a, s);
  if (a.vocab <= 16 * 256) return launch_plain<T, WIDE, 16, 256, 6>(a, s);
  if (a.vocab <= 32 * 256 * kProbsCtas) return launch_plain<T, WIDE, 32, 256, 4>(a, s);
  if (a.vocab <= 32 * 512 * kProbsCtas) return launch_plain<T, WIDE, 32, 512, 2>(a, s);
  return launch_plain<T, WIDE, 64, 512, 1>(a, s);
}
template <typename T>
cudaError_t launch_plain(const TokenProbsArgs& a, cudaStream_t s) {
  return rows_aligned<T>(a) ? launch_plain<T, true>(a, s) : launch_plain<T, false>(a, s);
}

}  // namespace

cudaError_t launch_probs_plain(const TokenProbsArgs& a, int dtype, cudaStream_t s) {
  return dtype == DVI_BF16 ? launch_plain<__nv_bfloat16>(a, s) : launch_plain<float>(a, s);
}

cudaError_t launch_token_probs(const TokenProbsArgs& a, int dtype, cudaStream_t s) {
  const bool cuts = a.top_k || a.top_p || a.top_p_all < 1.f || (a.top_k_all > 0 && a.top_k_all < a.vocab);
  if (!cuts) return launch_probs_plain(a, dtype, s);
  return a.vocab <= kShortRow ? launch_probs_short(a, dtype, s) : launch_probs_cut(a, dtype, s);
}

}  // namespace dvi
