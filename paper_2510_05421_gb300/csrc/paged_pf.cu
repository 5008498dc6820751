// Attention of many rows (prompt chunks, bf16) over the 8-bit paged cache on
// tcgen05 / TMEM; the formulas are those of paged_attn.cuh.
//
// A CTA owns one KV head and two tiles of 128 query vectors (tile row v: row
// v / G of the tile, query head v % G) and walks the 64-position chunks of
// the cache that its rows see.  Both tiles share every chunk, so the codes
// cross L2 and are widened to f16 once per 256 query vectors.  Per chunk and
// tile:
//   S = Q C_k^T    M = 128 vectors, N = 64 positions, K = hd (codes are exact
//                  in f16, and so are bf16 queries scaled by a power of two);
//   weights        one thread per vector: w = 2^(S f ks + log2 vs - m) as f16
//                  back into the TMEM columns of S, sum of w / vs;
//   O += W C_v     A = W from TMEM, B = the widened codes as they lie (rows are
//                  the K index: MN-major).
// The weights' f16 (2^-11 of each, as in paged_attn.cuh) is what the tensor operation
// takes beside f16 codes; the denominator sums them unrounded.  The accumulator is
// rescaled only when a vector's maximum outgrows its reference by 2^13.  A tile's scores are double-buffered in TMEM, two chunks
// ahead of the product of its weights, so its threads never wait for them.
//
// Roles (512 threads): warps 0-3 and 4-7 hold the vectors of tile 0 and 1,
// warps 8-11 widen codes (global -> registers -> SW128 tiles in shared memory,
// the next tile's codes in flight meanwhile), warp 12 issues the MMAs.
//
// Bound: 24 MMAs a chunk take 1290 cycles of the tensor pipe (the scores' are fed from
// shared memory at its rate) of the 2500 that the weights (1770) and the issuer's waits
// make of it.  Measured: 1000 rows behind 3001 positions, 32 heads of 128, int8 85.4 us
// (57.4 GFLOP, 0.67 PFLOP/s).
//
// Where the tiles are fewer than the SMs, `splits` CTAs share a pair of tiles
// along the positions; the last of them to end joins their parts in order.
//
// Every wait is bounded (flag, then wind down).
#include <algorithm>
#include <type_traits>

#include "paged.cuh"

namespace dvi {

namespace {

constexpr int kPfThreads = 512;
constexpr int kPfQ = 128;                // vectors per tile
constexpr int kPfPos = 64;               // positions per chunk
constexpr int kPfSegs = kPfPos / 16;     // a page covers whole segments
constexpr int kPfStages = 4;             // of K, and of V (even: a chunk's stage tells its score buffer)
constexpr float kPfLazy = 13.f;          // growth of a maximum that rescales the accumulator
constexpr float kPfUp = 5.f;             // a new reference sits so far below the maximum
constexpr float kPfUnset = -3e38f;       // the reference of a vector that has seen no key
constexpr float kPfLog2e = 1.4426950408889634f;
// What becomes of a product beside its scale: nothing; a bias or a cap; a large cap (see
// kPagedPlainCap; a kernel of its own, as the registers of both caps in one take the chunk of
// 1000 rows with a bias from 126 to 190 us).
constexpr int kPfStraight = 0, kPfCurved = 1, kPfFineCap = 2;

template <int HD>
struct PfSmem {
  static constexpr int kBoxes = HD / 64;               // 64-dim boxes per row
  static constexpr int kBox = kPfPos * 128;            // 64 rows x 64 f16
  static constexpr int kStage = kBoxes * kBox;         // one chunk's K or V
  static constexpr int kQBox = kPfQ * 128;
  static constexpr int kQ = kBoxes * kQBox;            // one tile's queries
  static constexpr int kRing = 2 * kQ;
  static constexpr int kFac = kRing + 2 * kPfStages * kStage;
  static constexpr int kBars = kFac + 2 * kPfQ * 4;
  static constexpr int kTotal = kBars + 256 + 1024 /*align*/;
};

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float lg2(float x) {
  float y;
  asm("lg2.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// Two f32 operations in one instruction.
__device__ __forceinline__ uint64_t pack2(float lo, float hi) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ float2 unpack2(uint64_t v) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
  return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
__device__ __forceinline__ uint32_t pack_h2(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
// Instruction descriptor of tcgen05.mma kind::f16 with f16 operands, M = 128.
__host__ __device__ constexpr uint32_t idesc_f16_m128(uint32_t n) {
  return (1u << 4) | ((n >> 3) << 17) | ((128u >> 4) << 24);
}
// Waits for this thread's TMEM loads, v's among them: the compiler cannot use v before.
__device__ __forceinline__ void tmem_ld_wait64(float (&v)[64]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
  for (int i = 0; i < 64; i += 8)
    asm volatile("" : "+f"(v[i]), "+f"(v[i + 1]), "+f"(v[i + 2]), "+f"(v[i + 3]), "+f"(v[i + 4]), "+f"(v[i + 5]),
                 "+f"(v[i + 6]), "+f"(v[i + 7]));
}
// One lane of a converged warp, always the same.
__device__ __forceinline__ bool elect_one() {
  uint32_t p;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(p));
  return p != 0;
}
// 16 codes as 16 f16.
template <bool E4M3>
__device__ __forceinline__ void widen(const uint4& q, uint4& lo, uint4& hi) {
  const uint32_t w[4] = {q.x, q.y, q.z, q.w};
  uint32_t h[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (E4M3) {
      e4m3x4_to_f16(w[i], h[2 * i], h[2 * i + 1]);
    } else {
      const uint32_t u = w[i] ^ 0x80808080u, c = 0x64806480u;     // 1152, 1152
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const uint32_t x = __byte_perm(u, 0x64646464u, k ? 0x4342 : 0x4140);
        const __half2 r = __hsub2(*reinterpret_cast<const __half2*>(&x), *reinterpret_cast<const __half2*>(&c));
        h[2 * i + k] = *reinterpret_cast<const uint32_t*>(&r);
      }
    }
  }
  lo = make_uint4(h[0], h[1], h[2], h[3]);
  hi = make_uint4(h[4], h[5], h[6], h[7]);
}

}  // namespace

template <bool E4M3, int HD, int CURVE>
__global__ void __launch_bounds__(kPfThreads, 1)
    paged_pf_kernel(const __grid_constant__ PagedAttendArgs a, int n_items, int rows_per_tile, int splits) {
  using SM = PfSmem<HD>;
  extern __shared__ uint8_t dsm_raw[];
  const uint32_t raw = smem_u32(dsm_raw);
  uint8_t* sm = dsm_raw + (((raw + 1023u) & ~1023u) - raw);
  float* fac = reinterpret_cast<float*>(sm + SM::kFac);
  uint64_t* full = reinterpret_cast<uint64_t*>(sm + SM::kBars);   // [K stages, V stages]
  uint64_t* empty = full + 2 * kPfStages;
  uint64_t* q_ready = empty + 2 * kPfStages;   // the queries are in shared memory
  uint64_t* s_full = q_ready + 1;          // [tile][2] the chunk's scores are in TMEM
  uint64_t* p_ready = s_full + 4;          // [tile][2] its weights are (made up to a chunk before they are used)
  uint64_t* pv_done = p_ready + 4;         // [2] its accumulator holds the chunk
  uint64_t* fin = pv_done + 2;             // every MMA issued is done
  uint32_t* tmem_holder = reinterpret_cast<uint32_t*>(fin + 1);
  int* last_s = reinterpret_cast<int*>(tmem_holder + 1);

  const PagedArgs& c = a.c;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int G = a.G, RT = rows_per_tile;
  auto row_of = [&](int v) { return G == 1 ? v : static_cast<int>(__umulhi(static_cast<uint32_t>(v), a.inv_g)); };   // v / G

  griddep_wait();
  griddep_launch();
  // ---------------- this CTA's item: a pair of tiles of one sequence (the last
  // pairs see most and go first), a KV head, a range of positions
  const int split = static_cast<int>(blockIdx.y);
  const int h = static_cast<int>(blockIdx.x) % c.H;
  const int item = n_items - 1 - static_cast<int>(blockIdx.x) / c.H;
  int first = 0;
  const int pair = 2 * RT;
  int b = 0;
  {
    auto begin = [&](int s) {
      const int r0 = c.row_start ? min(max(c.row_start[s], 0), c.n_rows) : s * (c.n_rows / c.n_seqs);
      return r0 / pair + s;
    };
    int n = 0;
    for (int s0 = 0; s0 < c.n_seqs; s0 += kPfThreads) {
      const int s = s0 + tid;
      n += __syncthreads_count(s < c.n_seqs && begin(s) <= item);
    }
    b = n - 1;
    if (b < 0) return;
    first = begin(b);
  }
  const PagedSeq sq = paged_seq(c, b);
  const int i0 = (item - first) * pair;                 // first row of tile 0
  const int vecs = sq.n * G;
  // (i0 < 0: row starts that do not ascend)
  if (i0 < 0 || i0 >= sq.n || vecs < a.min_vectors || vecs > a.max_vectors) return;
  const int cap = c.max_pages << c.log_p;
  const int held_end = min(sq.len + sq.n, cap);         // rows of the cache past it are nobody's
  // chunks that some row of tile t sees (0: the tile has no row), and those of this CTA
  auto seen = [&](int t) {
    const int nr = min(RT, sq.n - i0 - t * RT);
    return nr <= 0 ? 0 : (min(sq.len + i0 + t * RT + nr, cap) + kPfPos - 1) / kPfPos;
  };
  const int all0 = seen(0), all1 = seen(1), all = max(all0, all1);
  const int begin_all = min(a.window > 0 ? max(0, sq.len + i0 - a.window + 1) / kPfPos : 0, max(all - 1, 0));
  const int c0 = begin_all + (all - begin_all) * split / splits;
  const int c1 = begin_all + (all - begin_all) * (split + 1) / splits;
  const int nch0 = max(0, min(all0, c1) - c0), nch1 = max(0, min(all1, c1) - c0), nch = max(nch0, nch1);

  if (tid == 0) {
    for (int s = 0; s < 2 * kPfStages; ++s) {
      mbar_init(&full[s], 4);
      mbar_init(&empty[s], 1);
    }
    mbar_init(q_ready, 8);
    for (int t = 0; t < 2; ++t) {
      mbar_init(&s_full[2 * t], 1);
      mbar_init(&s_full[2 * t + 1], 1);
      mbar_init(&p_ready[2 * t], 4);
      mbar_init(&p_ready[2 * t + 1], 4);
      mbar_init(&pv_done[t], 1);
    }
    mbar_init(fin, 1);
    mbar_fence_init();
  }
  if (warp == 12) tmem_alloc(tmem_holder, 512);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_holder;
  // a split's part: [HD / 4][256 vectors] quads of dims, then maxima and sums
  constexpr int kPart = 2 * kPfQ * (HD + 2);
  const int unit = item * c.H + h;
  // S of tile t and chunk i: columns 128 t + 64 (i % 2) .., W over its first half; O: 256 + 128 t ..

  if (warp >= 12) {
    if (warp == 12) {
      // ---------------- MMA issuer: the whole warp walks the chunks and one lane issues.
      // The loop is unrolled over the stages, so that every descriptor is a uniform base
      // and a constant: with stages computed at run time an MMA took 107 cycles to issue
      // (54 on the pipe).
      const uint32_t id_s = idesc_f16_m128(kPfPos);
      const uint32_t id_o = idesc_f16_m128(HD) | kIdescBMn;
      const uint64_t q_desc = smem_desc_sw128(smem_u32(sm));
      const uint64_t k_desc = smem_desc_sw128(smem_u32(sm + SM::kRing));
      const uint64_t v_desc = smem_desc_sw128_mn(smem_u32(sm + SM::kRing + kPfStages * SM::kStage), SM::kBox);
      const uint32_t tm = __reduce_max_sync(0xffffffffu, tmem);
      // scores of tile t and a chunk whose stage is s (a multiple of 4 before it)
      auto scores = [&](int t, int s) {
        const uint64_t q = q_desc + static_cast<uint64_t>(t * (SM::kQ >> 4));
        const uint64_t k = k_desc + static_cast<uint64_t>(s * (SM::kStage >> 4));
        if (elect_one()) {
#pragma unroll
          for (int kk = 0; kk < HD / 16; ++kk)
            tc_mma_bf16(tm + 128u * t + 64u * (s & 1), q + ((kk / 4) * (SM::kQBox >> 4) + (kk % 4) * 2),
                        k + ((kk / 4) * (SM::kBox >> 4) + (kk % 4) * 2), id_s, kk != 0);
          tc_commit(&s_full[2 * t + (s & 1)]);
        }
        __syncwarp();
      };
      auto values = [&](int t, int s, uint32_t add) {
        const uint64_t v = v_desc + static_cast<uint64_t>(s * (SM::kStage >> 4));
        if (elect_one()) {
#pragma unroll
          for (int kk = 0; kk < kPfPos / 16; ++kk)
            tc_mma_bf16_ta(tm + 256u + 128u * t, tm + 128u * t + 64u * (s & 1) + 8u * kk, v + kk * (2048 >> 4), id_o,
                           kk == 0 ? add : 1u);
          tc_commit(&pv_done[t]);
        }
        __syncwarp();
      };
      auto release = [&](int kv, int s) {
        if (elect_one()) tc_commit(&empty[kv * kPfStages + s]);
        __syncwarp();
      };
      auto full_wait = [&](int kv, int i) {
        const bool r = mbar_wait(&full[kv * kPfStages + i % kPfStages], (i / kPfStages) & 1, c.status);
        tc_fence_after();
        return r;
      };
      bool ok = nch > 0 && mbar_wait(q_ready, 0, c.status);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        if (i >= nch || !ok) break;
        ok = full_wait(0, i);
        if (!ok) break;
        if (i < nch0) scores(0, i);
        if (i < nch1) scores(1, i);
        release(0, i);
      }
      // the scores are two chunks ahead of the weights' product, so the weights never wait for them
      for (int i4 = 0; i4 < nch && ok; i4 += kPfStages) {
#pragma unroll
        for (int s = 0; s < kPfStages; ++s) {
          const int i = i4 + s, s2 = (s + 2) % kPfStages;
          if (i >= nch || !ok) break;
          const bool more = i + 2 < nch;
          ok = full_wait(1, i) && (!more || full_wait(0, i + 2));
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            if (!ok || i >= (t ? nch1 : nch0)) continue;
            ok = mbar_wait(&p_ready[2 * t + (s & 1)], (i >> 1) & 1, c.status);
            if (!ok) continue;
            tc_fence_after();
            values(t, s, i > 0);
          }
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            if (!ok || i + 2 >= (t ? nch1 : nch0)) continue;
            // the scores of chunk i + 2 overwrite the columns that product i reads
            ok = mbar_wait(&pv_done[t], i & 1, c.status);
            if (!ok) continue;
            tc_fence_after();
            scores(t, s2);
          }
          if (!ok) break;
          release(1, s);
          if (more) release(0, s2);
        }
      }
      // every MMA issued is done before the TMEM is freed
      if (elect_one()) tc_commit(fin);
      mbar_wait(fin, 0, c.status);
    }
    __syncwarp();
  } else if (warp >= 8) {
    // ---------------- widening: tiles K c0, V c0, K c0 + 1, ...; a warp has the 16 rows of one segment
    const int w = warp - 8;
    constexpr int kRow = HD / 16;                       // 16-byte chunks of a row
    constexpr int kRows = 32 / kRow;                    // rows at once
    constexpr int kLoads = 16 / kRows;
    // eight lanes write two rows of one 64-dim box: no bank meets twice
    const int ch = HD == 128 ? (lane & 3) | ((lane >> 1) & 4) : lane & 3;
    const int r0 = HD == 128 ? ((lane >> 2) & 1) | ((lane >> 3) & 2) : lane >> 2;
    const size_t page_bytes = (static_cast<size_t>(c.H) << c.log_p) * HD;
    const size_t lane_off = ((static_cast<size_t>(h) << c.log_p) + r0) * HD + ch * 16;
    auto entry = [&](int i) {
      const int p = (c0 + i) * kPfPos + 16 * w;
      return i < nch && p < held_end ? paged_entry(c, b, p >> c.log_p) : -1;
    };
    // codes of two chunks are in flight: chunk i's in code[i % 2]
    uint4 code[2][2][kLoads];
    auto load = [&](int i, uint4 (&to)[2][kLoads], int raw_entry) {
      const int pg = paged_valid(c, raw_entry), p = (c0 + i) * kPfPos + 16 * w;
      const size_t at = static_cast<size_t>(max(pg, 0)) * page_bytes + (p & (c.P - 1)) * HD + lane_off;
      const int live = pg >= 0 ? held_end - p - r0 : 0;            // rows past it, and pages not held: zeros
#pragma unroll
      for (int kv = 0; kv < 2; ++kv)
#pragma unroll
        for (int u = 0; u < kLoads; ++u)
          to[kv][u] = u * kRows < live ? __ldg(reinterpret_cast<const uint4*>((kv ? c.v : c.k) + at + u * kRows * HD))
                                       : make_uint4(0u, 0u, 0u, 0u);
    };
    const int first_entry = entry(0), second_entry = entry(1);
    int ent = entry(2);
    if (nch > 0) load(0, code[0], first_entry);
    if (nch > 1) load(1, code[1], second_entry);
    bool ok = true;
    for (int i0w = 0; i0w < nch && ok; i0w += 2) {
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const int i = i0w + k;
        if (i >= nch || !ok) break;
        const int s = i % kPfStages;
#pragma unroll
        for (int kv = 0; kv < 2; ++kv) {
          ok = ok && mbar_wait(&empty[kv * kPfStages + s], ((i / kPfStages) & 1) ^ 1, c.status);
          if (!ok) break;
          uint8_t* dst = sm + SM::kRing + (kv * kPfStages + s) * SM::kStage + (ch / 4) * SM::kBox;
#pragma unroll
          for (int u = 0; u < kLoads; ++u) {
            uint4 x[2];
            widen<E4M3>(code[k][kv][u], x[0], x[1]);
#pragma unroll
            for (int e = 0; e < 2; ++e)
              *reinterpret_cast<uint4*>(dst + sw128_offset(16 * w + u * kRows + r0, (2 * (ch % 4) + e) * 8)) = x[e];
          }
          fence_proxy_async_smem();
          __syncwarp();
          if (lane == 0) mbar_arrive(&full[kv * kPfStages + s]);
        }
        if (ok && i + 2 < nch) load(i + 2, code[k], ent);
        ent = entry(i + 3);
      }
    }
  } else {
    // ---------------- a tile's vectors
    const int t = warp >> 2, wq = warp & 3;
    const int r0 = i0 + t * RT;
    const int nrows = max(0, min(RT, sq.n - r0));
    const int my = t ? nch1 : nch0;
    // thread = TMEM lane = vector
    const int v = wq * 32 + lane, vi = row_of(v), hq = h * G + v - vi * G;
    const bool live = vi < nrows;
    // The warp's queries, each scaled by a power of two to [2^14, 2^15): a row's 16-byte
    // pieces on neighbouring lanes, all rows in flight at once
    constexpr int kPieces = HD / 8, kRowsAtOnce = 32 / kPieces, kReads = 32 / kRowsAtOnce;
    const int piece = lane % kPieces, sub = lane / kPieces;
    {
      uint4 x[kReads];
#pragma unroll
      for (int i = 0; i < kReads; ++i) {
        const int vv = wq * 32 + i * kRowsAtOnce + sub, ii = row_of(vv);
        x[i] = make_uint4(0u, 0u, 0u, 0u);
        if (ii < nrows)
          x[i] = __ldg(reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(a.q) +
                                                      static_cast<long long>(sq.row0 + r0 + ii) * a.ld_q +
                                                      (h * G + vv - ii * G) * HD) + piece);
      }
      uint8_t* qs = sm + t * SM::kQ + (piece / 8) * SM::kQBox;
#pragma unroll
      for (int i = 0; i < kReads; ++i) {
        const int vv = wq * 32 + i * kRowsAtOnce + sub;
        const uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
        float top = 0.f;
#pragma unroll
        for (int e = 0; e < 4; ++e) top = max3(top, fabsf(bf16_lo(w[e])), fabsf(bf16_hi(w[e])));
#pragma unroll
        for (int o = kPieces / 2; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        const int ex = max(static_cast<int>(__float_as_uint(top) >> 23), 15);
        const float up = __uint_as_float(static_cast<uint32_t>(268 - ex) << 23);
        if (piece == 0) fac[t * kPfQ + vv] = __uint_as_float(static_cast<uint32_t>(ex - 14) << 23);
        uint32_t y[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = pack_h2(bf16_lo(w[e]) * up, bf16_hi(w[e]) * up);
        *reinterpret_cast<uint4*>(qs + sw128_offset(vv, (piece % 8) * 8)) = make_uint4(y[0], y[1], y[2], y[3]);
      }
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(q_ready);
    }
    const float down = fac[t * kPfQ + v];
    const float f = fmaxf(CURVE == kPfCurved && a.softcap > 0.f ? down * (a.scale / a.softcap)
                                                                : down * (a.scale * kPfLog2e), 1.2e-38f);
    const int pos = sq.len + r0 + vi;
    const float slope = a.slopes && live ? __ldg(a.slopes + hq) * kPfLog2e : 0.f;
    const uint32_t lanes = static_cast<uint32_t>(wq * 32) << 16;
    const uint32_t ts = tmem + 128u * t + lanes, to = tmem + 256u + 128u * t + lanes;
    // scales: lane e < 4 holds those of segment e; entries are read two chunks ahead, scales one
    auto entry = [&](int i) {
      const int p = (c0 + i) * kPfPos + 16 * lane;
      return lane < kPfSegs && i < my && p < held_end ? paged_entry(c, b, p >> c.log_p) : -1;
    };
    int e_next = entry(0);
    float ks_next = 0.f, vs_next = 0.f;
    auto scales = [&] {
      const int pg = paged_valid(c, e_next);
      ks_next = pg >= 0 ? __ldg(c.k_scale + static_cast<size_t>(pg) * c.H + h) : 0.f;
      vs_next = pg >= 0 ? __ldg(c.v_scale + static_cast<size_t>(pg) * c.H + h) : 0.f;
    };
    scales();
    e_next = entry(1);
    float m = kPfUnset, l = 0.f;
    bool ok = true;
#pragma unroll 1
    for (int i = 0; i < my; ++i) {
      const float vx = fmaxf(vs_next, kPagedMinScale);
      const float ks_l = vs_next > 0.f ? ks_next : 1.f, lv_l = vs_next > 0.f ? lg2(vx) : -INFINITY;
      const float iv_l = __fdividef(1.f, vx);
      scales();
      e_next = entry(i + 2);
      if (!mbar_wait(&s_full[2 * t + (i & 1)], (i >> 1) & 1, c.status)) {
        ok = false;
        break;
      }
      tc_fence_after();
      const uint32_t tsi = ts + 64u * (i & 1);
      const int at = (c0 + i) * kPfPos;
      const int see = pos - at;                        // positions 0 .. see of the chunk are visible,
      const int from = a.window > 0 ? see - a.window + 1 : 0;       // and only those from here on
      const bool edge = __any_sync(0xffffffffu, live && (see < kPfPos - 1 || from > 0));
      float s[kPfPos], fk[kPfSegs], lv[kPfSegs];
      tmem_ld32_async(tsi, s);
      tmem_ld32_async(tsi + 32, s + 32);
#pragma unroll
      for (int g = 0; g < kPfSegs; ++g) {
        fk[g] = fmaxf(f * __shfl_sync(0xffffffffu, ks_l, g), 1.2e-38f);   // not 0: a masked score stays -inf
        lv[g] = __shfl_sync(0xffffffffu, lv_l, g);
      }
      tmem_ld_wait64(s);
      if (CURVE != kPfStraight) {
        // the finished scores in place of the products
#pragma unroll
        for (int e = 0; e < kPfPos; ++e) {
          float x = s[e] * fk[e / 16];
          if (CURVE == kPfFineCap) x = paged_cap_fine(x, a.cap);
          else if (a.softcap > 0.f)
            x = (1.f - __fdividef(2.f, 1.f + ex2(x * (2.f * kPfLog2e)))) * (a.softcap * kPfLog2e);
          s[e] = fmaf(slope, static_cast<float>(e - see), x + lv[e / 16]);
        }
      }
      if (edge) {
#pragma unroll
        for (int e = 0; e < kPfPos; ++e) s[e] = e <= see && e >= from ? s[e] : -INFINITY;
      }
      float top = -INFINITY;
#pragma unroll
      for (int g = 0; g < kPfSegs; ++g) {
        const float* z = s + 16 * g;
        float x = fmaxf(z[0], z[1]), y = fmaxf(z[2], z[3]);
#pragma unroll
        for (int e = 4; e < 16; e += 4) x = max3(x, z[e], z[e + 1]), y = max3(y, z[e + 2], z[e + 3]);
        x = fmaxf(x, y);
        // a segment's factor is positive: its largest product is its largest score
        top = fmaxf(top, CURVE != kPfStraight ? x : fmaf(x, fk[g], lv[g]));
      }
      const bool move = top > m + kPfLazy;
      if (__any_sync(0xffffffffu, move)) {
        const float ref = move ? top - kPfUp : m, shrink = ex2(m - ref);
        m = ref;
        l *= shrink;
        if (i > 0) {
          if (!mbar_wait(&pv_done[t], (i - 1) & 1, c.status)) {
            ok = false;
            break;
          }
          tc_fence_after();
#pragma unroll 1
          for (int d = 0; d < HD; d += 16) {
            float o[16];
            tmem_ld16(to + d, o);
            uint32_t r[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) r[e] = __float_as_uint(o[e] * shrink);
            tmem_st16(to + d, r);
          }
          tmem_st_wait();
        }
      }
#pragma unroll
      for (int q = 0; q < kPfPos / 32; ++q) {
        uint32_t w[16];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const int g = 2 * q + k;
          // (the score is rounded as it is for the maximum, before the reference goes off)
          const uint64_t f2 = pack2(fk[g], fk[g]), l2 = pack2(lv[g], lv[g]), m2 = pack2(-m, -m);
          uint64_t sum = 0ull;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const uint64_t z = pack2(s[16 * g + 2 * e], s[16 * g + 2 * e + 1]);
            const float2 x = unpack2(add2(CURVE != kPfStraight ? z : fma2(z, f2, l2), m2));
            const float p0 = ex2(x.x), p1 = ex2(x.y);
            sum = add2(sum, pack2(p0, p1));
            w[8 * k + e] = pack_h2(p0, p1);
          }
          const float2 both = unpack2(sum);
          l = fmaf(both.x + both.y, __shfl_sync(0xffffffffu, iv_l, g), l);
        }
        tmem_st16(tsi + 16 * q, w);
      }
      tmem_st_wait();
      // A parity tells neighbouring phases apart only.  Chunk i's scores say that product
      // i - 2 is done; the wait for the last product, below, needs the one before it
      // done, and the last not begun, while this warp still holds its weights back.
      if (i + 1 == my && i > 0 && !mbar_wait(&pv_done[t], (i - 1) & 1, c.status)) {
        ok = false;
        break;
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&p_ready[2 * t + (i & 1)]);
    }
    // ---------------- O / l, or this split's part
    float* part = a.pf_part + static_cast<size_t>(unit * splits + split) * kPart;
    const bool done = ok && my > 0 && mbar_wait(&pv_done[t], (my - 1) & 1, c.status);
    if (done) tc_fence_after();
    const float inv = l > 0.f ? 1.f / l : (l == l ? 0.f : l);
    // (a vector whose weights were all 0 has an accumulator of zeros; a tile without chunks none at all)
    const int vp = t * kPfQ + v;
    // whole: the rows go through the tile's queries' place (every score is computed), so that
    // a row's pieces leave on neighbouring lanes
    uint8_t* os = sm + t * SM::kQ;
#pragma unroll 1
    for (int d = 0; d < HD; d += 16) {
      float o[16];
      if (done) tmem_ld16(to + d, o);
      else {
#pragma unroll
        for (int e = 0; e < 16; ++e) o[e] = 0.f;
      }
      if (splits == 1) {
        uint32_t w[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = pack_bf16x2(o[2 * e] * inv, o[2 * e + 1] * inv);
        uint8_t* at = os + (d / 64) * SM::kQBox;
        *reinterpret_cast<uint4*>(at + sw128_offset(v, d % 64)) = make_uint4(w[0], w[1], w[2], w[3]);
        *reinterpret_cast<uint4*>(at + sw128_offset(v, d % 64 + 8)) = make_uint4(w[4], w[5], w[6], w[7]);
      } else if (live) {
#pragma unroll
        for (int e = 0; e < 16; e += 4)
          __stcg(reinterpret_cast<float4*>(part + static_cast<size_t>((d + e) / 4) * (2 * kPfQ * 4) + vp * 4),
                 make_float4(o[e], o[e + 1], o[e + 2], o[e + 3]));
      }
    }
    if (splits == 1) {
      __syncwarp();
#pragma unroll 4
      for (int i = 0; i < kReads; ++i) {
        const int vv = wq * 32 + i * kRowsAtOnce + sub, ii = row_of(vv);
        if (ii < nrows)
          *(reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(a.o) + static_cast<long long>(sq.row0 + r0 + ii) * a.ld_o +
                                     (h * G + vv - ii * G) * HD) + piece) =
              *reinterpret_cast<const uint4*>(os + (piece / 8) * SM::kQBox + sw128_offset(vv, (piece % 8) * 8));
      }
    }
    if (splits > 1) {
      __stcg(part + 2 * kPfQ * HD + vp, m);
      __stcg(part + 2 * kPfQ * HD + 2 * kPfQ + vp, l);
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 12) {
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
  if (splits == 1) return;
  // ---------------- the last split to end joins all parts, in order
  if (tid == 0) {
    const int n = paged_arrive(a.pf_counters + unit);
    *last_s = n == splits - 1;
    if (n == splits - 1) a.pf_counters[unit] = 0;
  }
  __syncthreads();
  if (!*last_s) return;
  const float* parts = a.pf_part + static_cast<size_t>(unit * splits) * kPart;
  const int rows = min(pair, sq.n - i0), vecs0 = min(rows, RT) * G, vecs_all = vecs0 + max(rows - RT, 0) * G;
  // kItems quads of a thread at a time, kAtOnce parts of each in flight
  auto join = [&](auto items, auto at_once) {
    constexpr int kItems = decltype(items)::value, kAtOnce = decltype(at_once)::value;
    const int total = vecs_all * (HD / 4);
#pragma unroll 1
    for (int e0 = tid; e0 < total; e0 += kItems * kPfThreads) {
      float M[kItems], L[kItems];
      float4 acc[kItems];
      const float* at[kItems];
      int vp[kItems], quad[kItems];
#pragma unroll
      for (int u = 0; u < kItems; ++u) {
        const int e = min(e0 + u * kPfThreads, total - 1);
        quad[u] = e / vecs_all;
        const int x = e - quad[u] * vecs_all, t = x < vecs0 ? 0 : 1;
        vp[u] = t * kPfQ + x - t * vecs0;
        at[u] = parts + static_cast<size_t>(quad[u] * (2 * kPfQ) + vp[u]) * 4;
        M[u] = kPfUnset, L[u] = 0.f, acc[u] = make_float4(0.f, 0.f, 0.f, 0.f);
      }
#pragma unroll 1
      for (int s0 = 0; s0 < splits; s0 += kAtOnce) {
        float pm[kItems][kAtOnce], ps[kItems][kAtOnce];
        float4 o[kItems][kAtOnce];
#pragma unroll
        for (int u = 0; u < kItems; ++u)
#pragma unroll
          for (int k = 0; k < kAtOnce; ++k) {
            const size_t p = static_cast<size_t>(min(s0 + k, splits - 1)) * kPart;
            pm[u][k] = __ldcg(parts + p + 2 * kPfQ * HD + vp[u]);
            ps[u][k] = __ldcg(parts + p + 2 * kPfQ * HD + 2 * kPfQ + vp[u]);
            o[u][k] = __ldcg(reinterpret_cast<const float4*>(at[u] + p));
          }
#pragma unroll
        for (int u = 0; u < kItems; ++u) {
          float top = M[u];
#pragma unroll
          for (int k = 0; k < kAtOnce; ++k)
            if (s0 + k < splits) top = fmaxf(top, pm[u][k]);
          const float shrink = ex2(M[u] - top);
          M[u] = top;
          acc[u].x *= shrink, acc[u].y *= shrink, acc[u].z *= shrink, acc[u].w *= shrink, L[u] *= shrink;
#pragma unroll
          for (int k = 0; k < kAtOnce; ++k) {
            if (s0 + k >= splits) continue;
            const float w = ex2(pm[u][k] - top);
            acc[u].x = fmaf(o[u][k].x, w, acc[u].x), acc[u].y = fmaf(o[u][k].y, w, acc[u].y);
            acc[u].z = fmaf(o[u][k].z, w, acc[u].z), acc[u].w = fmaf(o[u][k].w, w, acc[u].w);
            L[u] = fmaf(ps[u][k], w, L[u]);
          }
        }
      }
#pragma unroll
      for (int u = 0; u < kItems; ++u) {
        if (e0 + u * kPfThreads >= total) continue;
        const int t = vp[u] / kPfQ, v = vp[u] % kPfQ, r = row_of(v), row = i0 + t * RT + r, hq = h * G + v - r * G;
        const float k = L[u] > 0.f ? 1.f / L[u] : (L[u] == L[u] ? 0.f : L[u]);
        *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(a.o) + static_cast<long long>(sq.row0 + row) * a.ld_o +
                                  hq * HD + 4 * quad[u]) =
            make_uint2(pack_bf16x2(acc[u].x * k, acc[u].y * k), pack_bf16x2(acc[u].z * k, acc[u].w * k));
      }
    }
  };
  using std::integral_constant;
  if (splits <= 3) join(integral_constant<int, 4>{}, integral_constant<int, 3>{});
  else join(integral_constant<int, 1>{}, integral_constant<int, 8>{});
}

namespace {

template <bool E4M3, int HD, int CURVE>
cudaError_t launch_pf(const PagedAttendArgs& a, int n_sms, cudaStream_t s) {
  static PerDevice attr;
  attr.once([] {
    cudaFuncSetAttribute(paged_pf_kernel<E4M3, HD, CURVE>, cudaFuncAttributeMaxDynamicSharedMemorySize, PfSmem<HD>::kTotal);
  });
  const PagedArgs& c = a.c;
  const int rt = kPfQ / a.G;
  const int per = c.row_start ? 0 : c.n_rows / c.n_seqs;
  // pairs of tiles: sequence b's begin at row_start[b] / (2 rt) + b
  const long long items = c.row_start ? c.n_rows / (2 * rt) + c.n_seqs
                                      : (static_cast<long long>(c.n_seqs - 1) * per) / (2 * rt) + c.n_seqs - 1 +
                                            (per + 2 * rt - 1) / (2 * rt);
  const long long units = items * c.H;
  if (units > 0x7fffffffll) return cudaErrorInvalidConfiguration;
  // splits only fill SMs that the tiles leave idle, eight chunks each at the least
  const int chunks = static_cast<int>(((static_cast<long long>(c.max_pages) << c.log_p) + kPfPos - 1) / kPfPos);
  const int splits = static_cast<int>(std::max(1ll, std::min<long long>({n_sms / units, chunks / 8, 16})));
  return launch_pdl(paged_pf_kernel<E4M3, HD, CURVE>, dim3(static_cast<unsigned>(units), splits), dim3(kPfThreads),
                    PfSmem<HD>::kTotal, s, a, static_cast<int>(items), rt, splits);
}

template <bool E4M3, int HD>
cudaError_t pf_scores(const PagedAttendArgs& a, int n_sms, cudaStream_t s) {
  if (a.cap.near > 0.f) return launch_pf<E4M3, HD, kPfFineCap>(a, n_sms, s);
  return a.softcap > 0.f || a.slopes ? launch_pf<E4M3, HD, kPfCurved>(a, n_sms, s)
                                     : launch_pf<E4M3, HD, kPfStraight>(a, n_sms, s);
}

}  // namespace

cudaError_t launch_paged_pf(const PagedAttendArgs& a, bool e4m3, int n_sms, cudaStream_t s) {
  if (a.c.D == 128) return e4m3 ? pf_scores<true, 128>(a, n_sms, s) : pf_scores<false, 128>(a, n_sms, s);
  return e4m3 ? pf_scores<true, 64>(a, n_sms, s) : pf_scores<false, 64>(a, n_sms, s);
}

}  // namespace dvi
