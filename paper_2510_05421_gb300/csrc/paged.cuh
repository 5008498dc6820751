// The 8-bit paged KV cache: what its kernels share.
//
// Codes lie in pages [n_pages][H_kv][P][D] (int8, or e4m3 bytes), one f32
// scale for each page and KV head: value = code * scale.  Sequence b's
// position p is row p % P of page table[b][p / P]; a negative entry is a page
// that is not held.  A call's rows of sequence b take the positions lens[b],
// lens[b] + 1, ...
#pragma once

#include <cuda_fp16.h>

#include "common.cuh"

namespace dvi {

constexpr int kPagedMaxSeqs = 1024;
constexpr float kPagedMinScale = 8.271806125530277e-25f;   // 2^-80

struct PagedArgs {
  uint8_t* k; uint8_t* v;
  float* k_scale; float* v_scale;
  const int* table; const int* lens; const int* row_start;
  int* status;
  int n_pages, H, P, log_p, D;
  int n_seqs, max_pages, n_rows, max_rows;
};

struct PagedAppendArgs {
  PagedArgs c;
  const void* kin; const void* vin; const void* q; void* q_out;
  long long ld_k, ld_v, ld_q, ld_qo;     // elements from row to row
  const float2* rotary;                   // [n_pos][rot / 2] (cos, sin); null: no rotation
  int rot, n_pos, n_heads, dtype;
};

struct PagedReadArgs {
  PagedArgs c;
  void* k_out; void* v_out;
  int dtype;
};

// c tanh(s / c) of scores in powers of two (x = s log2 e), for caps past kPagedPlainCap.
struct PagedCap {
  float inv;                              // 1 / (c log2 e)
  float two_inv;                          // 2 / c
  float top;                              // c log2 e
  float near;                             // |x| below it: by the series
};

struct PagedAttendArgs {
  PagedArgs c;
  const void* q; void* o;
  long long ld_q, ld_o;
  const float* slopes;                    // [n_heads] or null
  int n_heads, G, dtype;
  uint32_t inv_g;                         // ceil(2^32 / G): n / G = n inv_g >> 32 for small n (G = 1: 0, not used)
  float scale;
  float softcap;                          // c of f32 rows, and of bf16 rows up to kPagedPlainCap; 0: none
  PagedCap cap;                           // near > 0: that of bf16 rows under a larger one
  int window;                             // 0: none
  int min_vectors, max_vectors;           // sequences with rows * G in this range are this launch's
  int beside;                             // 1: the launch before is the same call's, on other rows: run beside it
  float* part;                            // partial results, then the counters
  int* counters;
  float* pf_part;                         // the same of the prompt kernel
  int* pf_counters;
};

cudaError_t launch_paged_append(const PagedAppendArgs& a, bool e4m3, cudaStream_t s);
cudaError_t launch_paged_read(const PagedReadArgs& a, bool e4m3, cudaStream_t s);
template <bool E4M3> cudaError_t launch_paged_attend(const PagedAttendArgs& a, int n_sms, cudaStream_t s);
cudaError_t launch_paged_pf(const PagedAttendArgs& a, bool e4m3, int n_sms, cudaStream_t s);

// Workspace of the attention: a counter for each team of warps (few rows) and
// for each pair of tiles (prompts), zero between calls, then two partial
// results of at most 32 vectors for each team, and one of 256 for each SM.
constexpr int kPagedTeams = 4;   // most teams per SM
inline size_t paged_counter_bytes(int n_sms) {
  return (static_cast<size_t>(n_sms) * (kPagedTeams + 1) * sizeof(int) + 255) / 256 * 256;
}
inline size_t paged_part_floats(int head_dim, int n_sms) {
  return static_cast<size_t>(n_sms) * kPagedTeams * 2 * 32 * (head_dim + 2);
}
inline size_t paged_pf_part_floats(int head_dim, int n_sms) {
  return static_cast<size_t>(n_sms) * 256 * (head_dim + 2);
}

// Counts one more part of a group in the workspace: how many came before.  What the
// block wrote before its barrier is released by it, and the others' parts acquired.
__device__ __forceinline__ int paged_arrive(int* counter) {
  int n;
  asm volatile("atom.add.acq_rel.gpu.global.s32 %0, [%1], 1;" : "=r"(n) : "l"(counter) : "memory");
  return n;
}

// tanh t = 1 - 2 / (1 + e^(2t)) in f32 is off by up to 2^-20 however small t is, a score capped
// so by that of the cap.  bf16 rows take it for caps up to kPagedPlainCap: the score is off by
// 2^-12, half of what a weight's rounding to f16 (2^-11 of it) is.  (f32 rows take tanhf.)
constexpr float kPagedPlainCap = 256.f;
// Under larger caps scores below a quarter of the cap go by the series of tanh up to t^7 (off by
// 3.3e-7 of themselves at t = 1/4) and only those beyond by the form above.  1000 rows behind
// 3001 positions, 32 heads of 128: 224 us so, 162 by the one form alone.
__device__ __forceinline__ float paged_cap_fine(float x, const PagedCap& c) {
  const float t = x * c.inv, u = t * t;
  float e;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(x * c.two_inv));
  return fabsf(x) < c.near ? fmaf(x * u, fmaf(u, fmaf(u, -17.f / 315.f, 2.f / 15.f), -1.f / 3.f), x)
                           : fmaf(-c.top, __fdividef(2.f, 1.f + e), c.top);
}

// ---------------------------------------------------------------- rows of a sequence
struct PagedSeq {
  int len;      // positions before the call's rows
  int row0;     // first row
  int n;        // rows
};
// Out-of-range row_start entries are cut to the call's rows, and a negative
// length counts as 0, so that no index leaves its buffer; both are flagged.
__device__ __forceinline__ PagedSeq paged_seq(const PagedArgs& c, int b) {
  PagedSeq s;
  s.len = c.lens[b];
  int r1;
  if (c.row_start) {
    s.row0 = c.row_start[b];
    r1 = c.row_start[b + 1];
  } else {
    const int per = c.n_rows / c.n_seqs;
    s.row0 = b * per;
    r1 = s.row0 + per;
  }
  s.n = r1 - s.row0;
  const int cap = c.max_pages << c.log_p;                         // the host refuses more than 2^30
  if (s.len < 0 || s.row0 < 0 || s.n < 0 || r1 > c.n_rows || s.n > c.max_rows || s.n > cap - s.len) {
    flag_status(c.status, DVI_DEV_KV_FULL);
    s.len = min(max(s.len, 0), cap);
    s.row0 = min(max(s.row0, 0), c.n_rows);
    s.n = min(min(max(s.n, 0), c.max_rows), c.n_rows - s.row0);
  }
  return s;
}
// A table entry as it lies there (a slot past the table: not held), and the
// page it names, or -1 where none is held.  Apart, so that entries can be in
// flight before the first of them is looked at.
__device__ __forceinline__ int paged_entry(const PagedArgs& c, int b, int slot) {
  return slot < c.max_pages ? __ldg(c.table + static_cast<size_t>(b) * c.max_pages + slot) : -1;
}
__device__ __forceinline__ int paged_valid(const PagedArgs& c, int entry) {
  if (entry < c.n_pages) return max(entry, -1);
  flag_status(c.status, DVI_DEV_KV_FULL);
  return -1;
}
__device__ __forceinline__ int paged_page(const PagedArgs& c, int b, int slot) {
  return paged_valid(c, paged_entry(c, b, slot));
}

// Work items of ragged sequences on a flat grid: sequence b owns the items
// from row_start[b] / unit + extra * b on, and has at most
// (n_b - 1) / unit + 1 + (extra - 1) of them, so no two sequences overlap.
// Every thread of the block calls it with the same item; -1: nobody's.
__device__ __forceinline__ int paged_seq_of_item(const PagedArgs& c, int item, int log_unit, int extra, int* first) {
  if (!c.row_start) {
    const int per = c.n_rows / c.n_seqs;
    auto begin = [&](int b) { return ((b * per) >> log_unit) + extra * b; };
    int b = static_cast<int>(__fdividef(static_cast<float>(item) * static_cast<float>(1 << log_unit),
                                        static_cast<float>(per) + static_cast<float>(extra << log_unit)));
    b = min(b, c.n_seqs - 1);
    while (b > 0 && begin(b) > item) --b;
    while (b + 1 < c.n_seqs && begin(b + 1) <= item) ++b;
    *first = begin(b);
    return b;
  }
  int n = 0;
  for (int b0 = 0; b0 < c.n_seqs; b0 += blockDim.x) {
    const int b = b0 + static_cast<int>(threadIdx.x);
    int begin = 0x7fffffff;
    if (b < c.n_seqs) begin = (min(max(c.row_start[b], 0), c.n_rows) >> log_unit) + extra * b;
    n += __syncthreads_count(begin <= item);
  }
  const int b = n - 1;
  if (b >= 0) *first = (min(max(c.row_start[b], 0), c.n_rows) >> log_unit) + extra * b;
  return b;
}

// ---------------------------------------------------------------- codes
template <bool E4M3> struct Code;
// int8: adding 1.5 * 2^23 rounds |x| < 2^22 to the nearest integer (ties to
// even) and leaves it in the low bits; the byte with its sign bit turned is
// code + 128, and 0x4b000000 | byte is the f32 number 2^23 + byte.
template <> struct Code<false> {
  static constexpr float kTop = 127.f;
  static __device__ __forceinline__ uint32_t enc4(float a, float b, float c, float d) {   // |x| < 128
    const float r = 12582912.f;
    const uint32_t ab = __byte_perm(__float_as_uint(__fadd_rn(a, r)), __float_as_uint(__fadd_rn(b, r)), 0x0040);
    const uint32_t cd = __byte_perm(__float_as_uint(__fadd_rn(c, r)), __float_as_uint(__fadd_rn(d, r)), 0x0040);
    return __byte_perm(ab, cd, 0x5410);
  }
  static __device__ __forceinline__ void dec4(uint32_t w, float (&x)[4]) {
    const uint32_t u = w ^ 0x80808080u;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      x[i] = __fsub_rn(__uint_as_float(__byte_perm(u, 0x4b000000u, 0x7440 | i)), 8388736.f);
  }
};
// Four e4m3 codes as two f16 pairs (exact).
__device__ __forceinline__ void e4m3x4_to_f16(uint32_t w, uint32_t& a, uint32_t& b) {
  asm("{\n\t.reg .b16 lo, hi;\n\tmov.b32 {lo, hi}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, lo;\n\t"
      "cvt.rn.f16x2.e4m3x2 %1, hi;\n\t}"
      : "=r"(a), "=r"(b)
      : "r"(w));
}
template <> struct Code<true> {
  static constexpr float kTop = 448.f;
  static __device__ __forceinline__ uint32_t enc2(float lo, float hi) {
    uint32_t r;
    asm("{\n\t.reg .b16 h;\n\tcvt.rn.satfinite.e4m3x2.f32 h, %2, %1;\n\tcvt.u32.u16 %0, h;\n\t}"
        : "=r"(r)
        : "f"(lo), "f"(hi));
    return r;
  }
  static __device__ __forceinline__ uint32_t enc4(float a, float b, float c, float d) {
    return enc2(a, b) | (enc2(c, d) << 16);
  }
  static __device__ __forceinline__ void dec4(uint32_t w, float (&x)[4]) {
    uint32_t lo, hi;
    e4m3x4_to_f16(w, lo, hi);
    const float2 a = __half22float2(*reinterpret_cast<const __half2*>(&lo));
    const float2 b = __half22float2(*reinterpret_cast<const __half2*>(&hi));
    x[0] = a.x, x[1] = a.y, x[2] = b.x, x[3] = b.y;
  }
};

// Eight consecutive elements, as they lie there and as f32.
template <typename T> struct Raw8;
template <> struct Raw8<float> {
  float4 a, b;
  __device__ __forceinline__ void load(const float* p) {
    a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
  }
  __device__ __forceinline__ void get(float (&x)[8]) const {
    x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
  }
};
template <> struct Raw8<__nv_bfloat16> {
  uint4 a;
  __device__ __forceinline__ void load(const __nv_bfloat16* p) { a = *reinterpret_cast<const uint4*>(p); }
  __device__ __forceinline__ void get(float (&x)[8]) const {
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) x[2 * i] = bf16_lo(w[i]), x[2 * i + 1] = bf16_hi(w[i]);
  }
};
template <typename T>
__device__ __forceinline__ void ld8(const T* p, float (&x)[8]) {
  Raw8<T> r;
  r.load(p);
  r.get(x);
}
__device__ __forceinline__ void st8(float* p, const float (&x)[8]) {
  reinterpret_cast<float4*>(p)[0] = make_float4(x[0], x[1], x[2], x[3]);
  reinterpret_cast<float4*>(p)[1] = make_float4(x[4], x[5], x[6], x[7]);
}
__device__ __forceinline__ void st8(__nv_bfloat16* p, const float (&x)[8]) {
  *reinterpret_cast<uint4*>(p) = make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]),
                                            pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7]));
}

}  // namespace dvi
