// Token probabilities: what the kernels for rows without and with cuts share.
#pragma once

#include <cooperative_groups.h>

#include "sample.cuh"

namespace dvi {

namespace cg = cooperative_groups;

constexpr int kProbsCtas = 8;   // most CTAs of a row

cudaError_t launch_probs_plain(const TokenProbsArgs& a, int dtype, cudaStream_t s);
cudaError_t launch_probs_cut(const TokenProbsArgs& a, int dtype, cudaStream_t s);
constexpr int kShortRow = 2048;   // most logits of a row for:
cudaError_t launch_probs_short(const TokenProbsArgs& a, int dtype, cudaStream_t s);

// log2(e) / T as an f32 pair, T within 2^-100 .. 2^100: the quotient's rest is exact by a fused
// multiply-add.
struct Slope {
  float hi, lo;
  __device__ __forceinline__ explicit Slope(float T) {
    const float t = fminf(fmaxf(T, 0x1p-100f), 0x1p100f), log2e = 0x1.715476p+0f, rest = 0x1.4ae0c0p-26f;
    hi = __fdiv_rn(log2e, t);
    lo = __fdiv_rn(fmaf(-hi, t, log2e) + rest, t);
  }
  // The same with hi below the whole and lo above 0.
  __device__ __forceinline__ Slope below() const {
    Slope s = *this;
    if (!(lo > 0.f)) {
      s.hi = __uint_as_float(__float_as_uint(hi) - 1);
      s.lo = lo + (hi - s.hi);
    }
    return s;
  }
};

// w in f32, by Slope::below (so both products of an infinite distance are -inf).  With c.hi alone its rounding would
// grow with the distance to the maximum, to one side; both halves' products are rounded together (576 rows of 32000
// without cuts 29.5 -> 30.0 us, of bf16 29.8 -> 31.3, with cuts 1 %).  x - m and the sum of the products stay rounded to
// 32 bits, either way: 2 units of 2^-24 for each unit of (m - x) / T at most.
__device__ __forceinline__ float weight(float x, float m, Slope c) {
  const float d = x - m;
  return exp2f(fmaf(d, c.hi, d * c.lo));
}

// A logit as it counts: NaN as -inf, +inf as the largest number, -0 as 0.
__device__ __forceinline__ float clean(float v) { return v != v ? -INFINITY : fminf(v, 3.402823466e38f) + 0.f; }

// f32 as a number that grows with it, and back.
__device__ __forceinline__ uint32_t ord(float x) {
  const uint32_t b = __float_as_uint(x);
  return (b & 0x80000000u) ? ~b : (b | 0x80000000u);
}
__device__ __forceinline__ float from_ord(uint32_t o) {
  return __uint_as_float((o & 0x80000000u) ? (o & 0x7fffffffu) : ~o);
}

// 16 bytes of logits.
__device__ __forceinline__ void load16(const float* p, float* v) {
  const float4 q = *reinterpret_cast<const float4*>(p);
  v[0] = q.x, v[1] = q.y, v[2] = q.z, v[3] = q.w;
}
__device__ __forceinline__ void load16(const __nv_bfloat16* p, float* v) {
  const uint4 q = *reinterpret_cast<const uint4*>(p);
  const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) v[2 * i] = bf16_lo(w[i]), v[2 * i + 1] = bf16_hi(w[i]);
}

// Whether rows are of whole 16 bytes and start on their boundaries, on both sides.
template <typename T>
bool rows_aligned(const TokenProbsArgs& a) {
  return a.vocab % (16 / sizeof(T)) == 0 && reinterpret_cast<uintptr_t>(a.x) % 16 == 0 && reinterpret_cast<uintptr_t>(a.out) % 16 == 0 &&
         (a.n_rows == 1 || (a.ld * sizeof(T) % 16 == 0 && a.ld_out % 4 == 0));
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

__device__ __forceinline__ void cluster_barrier(int n_ctas) {
  if (n_ctas > 1) {
    cluster_arrive_release();
    cluster_wait_acquire();
  } else {
    __syncthreads();
  }
}

// Eight bytes to the same place of CTA `rank`, counted by its barrier: no fence goes with them, so
// nothing waits for the sender's own memory operations.
__device__ __forceinline__ void send_to(void* to, unsigned long long v, void* bar, int rank) {
  asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.b64 [%0], %1, [%2];" ::"r"(
                   mapa_shared(smem_u32(to), rank)),
               "l"(v), "r"(mapa_shared(smem_u32(bar), rank))
               : "memory");
}
__device__ __forceinline__ unsigned long long bits_of(float a, float b) {
  return (static_cast<unsigned long long>(__float_as_uint(b)) << 32) | __float_as_uint(a);
}

// A cluster of `ctas` CTAs for each row, which hold slices of it.
template <typename K>
cudaError_t launch_rows(K kern, const TokenProbsArgs& a, int ctas, int threads, size_t smem, size_t smem_a_logit,
                        cudaStream_t s) {
  if (static_cast<int64_t>(a.n_rows) * ctas > 0x7fffffffll) return cudaErrorInvalidConfiguration;
  const int slice = ((a.vocab + ctas - 1) / ctas + 7) / 8 * 8;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(a.n_rows) * ctas);
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem + slice * smem_a_logit;
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

}  // namespace dvi
