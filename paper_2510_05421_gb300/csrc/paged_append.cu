// Rows into the 8-bit paged cache, and rows of it back as values.
//
// Append: k' = rot(k, p) in f32 (products and sums rounded one by one), then
// for each (page, KV head) that the call's rows touch
//   s = max(max |x| * (1 / Q), 2^-80)      Q = 127 (int8) or 448 (e4m3)
//   s = max(s, s_old)                      where earlier rows lie in the page
//   code = sat(rne(x * (1 / s)))
// and where s > s_old the earlier rows become rne(code * (s_old / s)).  A
// rolled-back row leaves its share in s, never in a value.  NaN is stored as
// 0 and an infinity as the largest code (both flagged), so that no cached
// value can reach another row through a probability of 0.
//
// A team of 32 to 256 threads owns one page of one head of K or of V: its
// rows are loaded and rotated once, 16 elements a thread and item (8 and their
// 8 rotation partners), and wait in registers for the page's maximum; its page
// entry is looked up meanwhile.  Two items a thread keep a thread within 64
// registers, so four blocks of 256 an SM hide each other's chain of loads
// (lengths, rows and entry, scale); only pages of 128 rows of hd 128 take four.
// Bound: bytes (the rows in, half or a quarter of them out).  8192 rows of 32 K,
// V and query heads each, e4m3 pages of 16: 73 to 75 us, 4.5 TB/s (83.4 with four
// items and two blocks; the 64 registers spill 12 to 32 bytes); 64 sequences' single tokens
// 5.6 us, one 2.8 us: latency.
#include <algorithm>

#include "paged.cuh"

namespace dvi {

namespace {

constexpr int kApThreads = 256;

// The (cos, sin) pairs of 8 dims.
struct Turn {
  float4 w[4];
  __device__ __forceinline__ void load(const float2* cs) {
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = __ldg(reinterpret_cast<const float4*>(cs) + i);
  }
};
__device__ __forceinline__ void rotate8(float (&a)[8], float (&b)[8], const Turn& t) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float co = i & 1 ? t.w[i >> 1].z : t.w[i >> 1].x, si = i & 1 ? t.w[i >> 1].w : t.w[i >> 1].y;
    const float x = __fsub_rn(__fmul_rn(a[i], co), __fmul_rn(b[i], si));
    const float y = __fadd_rn(__fmul_rn(b[i], co), __fmul_rn(a[i], si));
    a[i] = x;
    b[i] = y;
  }
}

// Element offsets of item j of a row: 8 elements and their 8 partners (the
// rotated dims first, then the others in the same halves).
__device__ __forceinline__ void item_dims(int j, int rot, int D, int& a, int& b) {
  if (8 * j < rot / 2) {
    a = 8 * j;
    b = a + rot / 2;
  } else {
    a = rot + 8 * j - rot / 2;
    b = a + (D - rot) / 2;
  }
}

template <int TEAM>
__device__ __forceinline__ float team_max(float v, float* red, int team, int t) {
  v = warp_max(v);
  if (TEAM == 32) return v;
  const int w = t >> 5;
  if ((t & 31) == 0) red[team * (TEAM / 32) + w] = v;
  named_bar(1 + team, TEAM);
#pragma unroll
  for (int i = 0; i < TEAM / 32; ++i) v = fmaxf(v, red[team * (TEAM / 32) + i]);
  return v;
}

template <bool E4M3, int D, typename T, int TEAM, int kApItems>
__device__ void append_page(const PagedAppendArgs& a, int item, int group) {
  __shared__ float red[kApThreads / 32];
  const PagedArgs& c = a.c;
  int first = 0;
  const int b = paged_seq_of_item(c, item, c.log_p, 2, &first);
  if (b < 0) return;
  const PagedSeq sq = paged_seq(c, b);
  const int slot = (sq.len >> c.log_p) + item - first;
  const int page0 = slot << c.log_p;                              // position of the page's row 0
  const int p0 = max(sq.len, page0), p1 = min(sq.len + sq.n, page0 + c.P);
  const int team = threadIdx.x / TEAM, t = threadIdx.x % TEAM;
  const int task = group * (kApThreads / TEAM) + team;
  if (p0 >= p1 || task >= 2 * c.H) return;                        // uniform over a team
  const bool is_v = task >= c.H;
  const int h = is_v ? task - c.H : task;
  const T* in = static_cast<const T*>(is_v ? a.vin : a.kin) + h * D;
  const long long ld = is_v ? a.ld_v : a.ld_k;
  const int rot = is_v ? 0 : a.rot;
  constexpr int kPer = D / 16;                                    // items of a row
  static_assert(TEAM % kPer == 0, "a thread's dims are the same in all its rows");
  const int n_items = (p1 - p0) * kPer, j = t % kPer;
  int da, db;
  item_dims(j, rot, D, da, db);
  // the rows do not wait for the page: both are in flight together
  const int entry = paged_entry(c, b, slot);
  Raw8<T> raw[kApItems][2];
#pragma unroll
  for (int u = 0; u < kApItems; ++u) {
    const int it = u * TEAM + t;
    if (it >= n_items) continue;
    const T* row = in + static_cast<long long>(sq.row0 + p0 - sq.len + it / kPer) * ld;
    raw[u][0].load(row + da);
    raw[u][1].load(row + db);
  }
  const int page = paged_valid(c, entry);
  if (page < 0) {
    if (t == 0) flag_status(c.status, DVI_DEV_KV_FULL);
    return;
  }
  const size_t ph = static_cast<size_t>(page) * c.H + h;
  float* sp = (is_v ? c.v_scale : c.k_scale) + ph;
  uint8_t* codes = (is_v ? c.v : c.k) + (ph << c.log_p) * D;
  const int held = p0 - page0;
  const float old = held > 0 ? *sp : 0.f;
  float x[kApItems][16];
  float most = 0.f, odd = 0.f;                                    // odd: NaN where some value is not finite
#pragma unroll
  for (int u = 0; u < kApItems; ++u) {
    const int it = u * TEAM + t;
    if (it >= n_items) continue;
    float lo[8], hi[8];
    raw[u][0].get(lo);
    raw[u][1].get(hi);
    if (8 * j < rot / 2) {
      const int pos = p0 + it / kPer;
      if (pos < a.n_pos) {
        Turn turn;
        turn.load(a.rotary + static_cast<size_t>(pos) * (rot / 2) + 8 * j);
        rotate8(lo, hi, turn);
      } else if (j == 0) {
        flag_status(c.status, DVI_DEV_KV_FULL);
      }
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const float v = i < 8 ? lo[i & 7] : hi[i & 7];
      most = fmaxf(most, fabsf(v));
      odd = fmaf(v, 0.f, odd);
      x[u][i] = v;
    }
  }
  if (odd != odd) {
    // NaN becomes 0, an infinity the largest code; neither counts for the scale
    flag_status(c.status, DVI_DEV_NONFINITE);
    most = 0.f;
#pragma unroll
    for (int u = 0; u < kApItems; ++u) {
      if (u * TEAM + t >= n_items) continue;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        if (x[u][i] != x[u][i]) x[u][i] = 0.f;
        else if (fabsf(x[u][i]) <= 3.402823466e38f) most = fmaxf(most, fabsf(x[u][i]));
      }
    }
  }
  most = team_max<TEAM>(most, red, team, t);
  float s = fmaxf(__fmul_rn(most, 1.f / Code<E4M3>::kTop), kPagedMinScale);
  if (held > 0) s = fmaxf(s, old);
  __syncwarp();   // the team has read the old scale (a larger team: by its barrier)
  if (t == 0) *sp = s;
  const float inv = __fdiv_rn(1.f, s);
#pragma unroll
  for (int u = 0; u < kApItems; ++u) {
    const int it = u * TEAM + t;
    if (it >= n_items) continue;
    uint8_t* row = codes + static_cast<size_t>(held + it / kPer) * D;
    float y[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) y[i] = __fmul_rn(x[u][i], inv);
    if (odd != odd) {
#pragma unroll
      for (int i = 0; i < 16; ++i) y[i] = fminf(fmaxf(y[i], -Code<E4M3>::kTop), Code<E4M3>::kTop);
    }
    using C = Code<E4M3>;
    *reinterpret_cast<uint2*>(row + da) = make_uint2(C::enc4(y[0], y[1], y[2], y[3]), C::enc4(y[4], y[5], y[6], y[7]));
    *reinterpret_cast<uint2*>(row + db) =
        make_uint2(C::enc4(y[8], y[9], y[10], y[11]), C::enc4(y[12], y[13], y[14], y[15]));
  }
  if (held > 0 && s > old) {
    const float f = __fdiv_rn(old, s);
    uint4* w = reinterpret_cast<uint4*>(codes);
    for (int i = t; i < held * kPer; i += TEAM) {
      const uint4 q = w[i];
      const uint32_t in4[4] = {q.x, q.y, q.z, q.w};
      uint32_t out4[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float v[4];
        Code<E4M3>::dec4(in4[e], v);
        out4[e] = Code<E4M3>::enc4(__fmul_rn(v[0], f), __fmul_rn(v[1], f), __fmul_rn(v[2], f), __fmul_rn(v[3], f));
      }
      w[i] = make_uint4(out4[0], out4[1], out4[2], out4[3]);
    }
  }
}

// Queries: a warp takes one row and `steps` * 32 items of its heads; a lane's
// dims are the same in every head, so it reads its (cos, sin) once.
template <int D, typename T>
__device__ void rotate_queries(const PagedAppendArgs& a, int warp_task, int parts, int steps) {
  const PagedArgs& c = a.c;
  const int lane = threadIdx.x & 31;
  const int r = warp_task / parts, part = warp_task % parts;
  if (r >= c.n_rows) return;
  int b;
  if (c.row_start) {
    int n = 0;
    for (int b0 = 0; b0 < c.n_seqs; b0 += 32) {
      const int e = b0 + lane;
      n += __popc(__ballot_sync(0xffffffffu, e < c.n_seqs && c.row_start[e] <= r));
    }
    b = n - 1;
  } else {
    b = r / (c.n_rows / c.n_seqs);
  }
  if (b < 0) return;
  const PagedSeq sq = paged_seq(c, b);
  const int i = r - sq.row0;
  if (i < 0 || i >= sq.n) return;
  const int pos = sq.len + i;
  constexpr int kPer = D / 16;
  const int j = lane % kPer, total = a.n_heads * kPer;
  int da, db;
  item_dims(j, a.rot, D, da, db);
  const bool turns = 8 * j < a.rot / 2 && pos < a.n_pos;
  if (pos >= a.n_pos && a.rot > 0 && lane == 0) flag_status(c.status, DVI_DEV_KV_FULL);
  Turn turn;
  if (turns) turn.load(a.rotary + static_cast<size_t>(pos) * (a.rot / 2) + 8 * j);
  const T* row = static_cast<const T*>(a.q) + static_cast<long long>(r) * a.ld_q;
  T* out = static_cast<T*>(a.q_out) + static_cast<long long>(r) * a.ld_qo;
#pragma unroll 4
  for (int u = part * steps; u < (part + 1) * steps; ++u) {
    const int it = u * 32 + lane;
    if (it >= total) break;
    const int h = it / kPer * D;
    float lo[8], hi[8];
    ld8(row + h + da, lo);
    ld8(row + h + db, hi);
    if (turns) rotate8(lo, hi, turn);
    st8(out + h + da, lo);
    st8(out + h + db, hi);
  }
}

template <bool E4M3, int D, typename T, int TEAM, int kApItems>
__global__ void __launch_bounds__(kApThreads, kApItems == 2 ? 4 : 2) paged_append_kernel(const __grid_constant__ PagedAppendArgs a,
                                                                  int n_items, int groups, int parts, int steps) {
  griddep_wait();
  griddep_launch();
  const int bid = static_cast<int>(blockIdx.x);
  const int pages = n_items * groups;
  if (bid < pages) append_page<E4M3, D, T, TEAM, kApItems>(a, bid / groups, bid % groups);
  else rotate_queries<D, T>(a, (bid - pages) * (kApThreads / 32) + static_cast<int>(threadIdx.x >> 5), parts, steps);
}

template <bool E4M3, int D, typename T, int TEAM, int kApItems>
cudaError_t launch_append(const PagedAppendArgs& a, cudaStream_t s) {
  const PagedArgs& c = a.c;
  const long long n_items = static_cast<long long>(c.n_rows >> c.log_p) + 2ll * c.n_seqs;
  const int teams = kApThreads / TEAM, groups = (2 * c.H + teams - 1) / teams;
  // a warp for all heads of a row where the rows alone fill the GPU, else for 64 items
  const int all_steps = (a.n_heads * (D / 16) + 31) / 32;
  const int steps = c.n_rows >= 4096 ? std::min(all_steps, 16) : std::min(all_steps, 2);
  const int parts = a.q ? (all_steps + steps - 1) / steps : 0;
  const long long q_blocks = (static_cast<long long>(c.n_rows) * parts + kApThreads / 32 - 1) / (kApThreads / 32);
  const long long blocks = n_items * groups + q_blocks;
  if (blocks > 0x7fffffffll) return cudaErrorInvalidConfiguration;
  return launch_pdl(paged_append_kernel<E4M3, D, T, TEAM, kApItems>, dim3(static_cast<unsigned>(blocks)), dim3(kApThreads), 0, s,
                    a, static_cast<int>(n_items), groups, parts, steps);
}
// A team's items are the rows of one page, as far as one sequence's rows go.
template <bool E4M3, int D, typename T>
cudaError_t append_teams(const PagedAppendArgs& a, cudaStream_t s) {
  const int items = std::min(a.c.P, a.c.max_rows) * (D / 16);
  if (items <= 64) return launch_append<E4M3, D, T, 32, 2>(a, s);
  if (items <= 128) return launch_append<E4M3, D, T, 64, 2>(a, s);
  if (items <= 256) return launch_append<E4M3, D, T, 128, 2>(a, s);
  if (items <= 512) return launch_append<E4M3, D, T, 256, 2>(a, s);
  return launch_append<E4M3, D, T, 256, 4>(a, s);
}
template <bool E4M3>
cudaError_t append_types(const PagedAppendArgs& a, cudaStream_t s) {
  if (a.dtype == DVI_BF16)
    return a.c.D == 128 ? append_teams<E4M3, 128, __nv_bfloat16>(a, s) : append_teams<E4M3, 64, __nv_bfloat16>(a, s);
  return a.c.D == 128 ? append_teams<E4M3, 128, float>(a, s) : append_teams<E4M3, 64, float>(a, s);
}

// ---------------------------------------------------------------- read
// A warp copies 16 positions (never more than a page) of one KV head of K or
// V, all its codes in flight at once; a block takes kRdWarps such tasks of the
// same positions.  Bound: bytes.  16384 positions of 32 heads of 128, e4m3 to bf16
// 69.8 us, 5.8 TB/s.
constexpr int kRdWarps = 8, kRdLog = 4;

template <bool E4M3, int D, typename T>
__global__ void __launch_bounds__(kRdWarps * 32) paged_read_kernel(const __grid_constant__ PagedReadArgs a, int groups) {
  griddep_wait();
  griddep_launch();
  const PagedArgs& c = a.c;
  const int item = static_cast<int>(blockIdx.x) / groups, group = static_cast<int>(blockIdx.x) % groups;
  int first = 0;
  const int b = paged_seq_of_item(c, item, kRdLog, 2, &first);
  if (b < 0) return;
  const PagedSeq sq = paged_seq(c, b);
  const int slot = (sq.len >> kRdLog) + item - first;
  const int begin = slot << kRdLog;
  const int p0 = max(sq.len, begin), p1 = min(sq.len + sq.n, begin + (1 << kRdLog));
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int task = group * kRdWarps + warp;
  if (p0 >= p1 || task >= 2 * c.H) return;
  const bool is_v = task >= c.H;
  const int h = is_v ? task - c.H : task;
  const int page = paged_page(c, b, p0 >> c.log_p);
  const size_t ph = static_cast<size_t>(max(page, 0)) * c.H + h;
  constexpr int kPer = D / 16, kSteps = (16 << kRdLog) * kPer / 16 / 32;
  const uint4* codes = reinterpret_cast<const uint4*>((is_v ? c.v : c.k) +
                                                      ((ph << c.log_p) + static_cast<size_t>(p0 & (c.P - 1))) * D);
  const int n = (p1 - p0) * kPer;
  uint4 q[kSteps];
#pragma unroll
  for (int u = 0; u < kSteps; ++u) {
    const int i = u * 32 + lane;
    q[u] = page >= 0 && i < n ? __ldg(codes + i) : make_uint4(0u, 0u, 0u, 0u);
  }
  const float s = page < 0 ? 0.f : (is_v ? c.v_scale : c.k_scale)[ph];
  T* out = static_cast<T*>(is_v ? a.v_out : a.k_out) + (static_cast<size_t>(sq.row0 + p0 - sq.len) * c.H + h) * D;
#pragma unroll
  for (int u = 0; u < kSteps; ++u) {
    const int i = u * 32 + lane;
    if (i >= n) break;
    const uint32_t w[4] = {q[u].x, q[u].y, q[u].z, q[u].w};
    float x[2][8];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float v[4];
      Code<E4M3>::dec4(w[e], v);
#pragma unroll
      for (int f = 0; f < 4; ++f) x[e >> 1][(e & 1) * 4 + f] = __fmul_rn(v[f], s);
    }
    T* dst = out + static_cast<size_t>(i / kPer) * c.H * D + 16 * (i % kPer);
    st8(dst, x[0]);
    st8(dst + 8, x[1]);
  }
}

template <bool E4M3, int D, typename T>
cudaError_t launch_read(const PagedReadArgs& a, cudaStream_t s) {
  const PagedArgs& c = a.c;
  const int groups = (2 * c.H + kRdWarps - 1) / kRdWarps;
  const long long blocks = (static_cast<long long>(c.n_rows >> kRdLog) + 2ll * c.n_seqs) * groups;
  if (blocks > 0x7fffffffll) return cudaErrorInvalidConfiguration;
  return launch_pdl(paged_read_kernel<E4M3, D, T>, dim3(static_cast<unsigned>(blocks)), dim3(kRdWarps * 32), 0, s, a,
                    groups);
}
template <bool E4M3>
cudaError_t read_types(const PagedReadArgs& a, cudaStream_t s) {
  if (a.dtype == DVI_BF16)
    return a.c.D == 128 ? launch_read<E4M3, 128, __nv_bfloat16>(a, s) : launch_read<E4M3, 64, __nv_bfloat16>(a, s);
  return a.c.D == 128 ? launch_read<E4M3, 128, float>(a, s) : launch_read<E4M3, 64, float>(a, s);
}

}  // namespace

cudaError_t launch_paged_append(const PagedAppendArgs& a, bool e4m3, cudaStream_t s) {
  return e4m3 ? append_types<true>(a, s) : append_types<false>(a, s);
}
cudaError_t launch_paged_read(const PagedReadArgs& a, bool e4m3, cudaStream_t s) {
  return e4m3 ? read_types<true>(a, s) : read_types<false>(a, s);
}

}  // namespace dvi
