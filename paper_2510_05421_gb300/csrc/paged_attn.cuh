// Attention of few rows over the 8-bit paged cache: decode rows and verify
// blocks (any number of rows is right; prompt chunks have a kernel of their
// own).
//
//   s_ij = (q_i . c_j) scale ks      s = cap tanh(s / cap)      s += slope (p_j - p_i)
//   o_i  = sum_j w_ij c_j / sum_j (w_ij / vs)       w_ij = 2^(s_ij log2 e + log2 vs - m_i)
// over the held positions p_i - window < p_j <= p_i.  Folding vs into the
// exponent keeps w in f16's range whatever the scales are, and the codes
// enter both products as they are (int8 and e4m3 values are exact in f16).
//
// The query vectors of one KV head (rows x its G query heads, 8 NT to a tile)
// are the columns of both products (warp MMAs, K and V as the row operand):
// the 16 x 16 K fragment takes 4 consecutive codes of a key per thread and
// step, any order of the dims being one, and the V fragment 16 consecutive
// codes of a key; the codes are loaded 16 bytes at a time and go to f16 in
// registers (1.25 to 1.5 instructions a code).
//
// Bound: bytes (the codes, read once) where few SMs' worth of ALU work is enough,
// the ALU at 16 vectors of int8 (widening is 112 of about 200 of its instructions
// a block).  Measured: 32 sequences of 12000 to 16384 positions, 12 vectors, 8 KV
// heads of 128, int8 165 us (932 MB, 5.6 TB/s); 9 rows over 16384, 32 heads of 128,
// int8 38.4 us (134 MB); 8 sequences up to 2560, 32 heads of 128, one row, e4m3
// 22.2 us (88 MB).  Beside its length a call costs about 7 us: lengths, plan, table
// entries, codes, joins, each waiting for the one before.
//
// Work: blocks of 16 positions.  The blocks of all (sequence, KV head, tile)
// groups lie in one row and every team of 4 to 16 warps takes an equal share of
// it, so ragged batches fill the GPU evenly; a group cut by shares is joined
// by whichever of its teams ends last, in the order of the shares (the result
// does not depend on which that is).  Inside a team the warps take blocks in
// turn, each with its own running maximum and a private ring of cp.async
// stages, and are joined in shared memory at the end of the group.
//
// Fewer bits than 32, and why: w goes to f16 for the tensor operation (2^-11 of it,
// and its error averages over the keys: below the 2^-8 of a bf16 result, measured
// against 64 bits the same as f32 arithmetic throughout); the denominator sums it
// unrounded.  f32 queries (PAIR) enter as an f16 pair hi + lo, as do their
// weights: 2^-21.  A query vector is scaled by a power of two so that f16's
// range does not matter.  log2 vs shares the exponent's f32 with the score: near
// the smallest vs (2^-80) its rounding is 2^-18 of the weight.
#pragma once

#include <algorithm>

#include "paged.cuh"

namespace dvi {

namespace {

constexpr int kPaKeys = 16;               // positions per block: never more than a page
constexpr int kPaTeam = 4;                // warps of the smallest team
constexpr int kPaOver = 4;                // steps of a warp that a group costs beside its blocks
constexpr float kPaLazy = 8.f;            // growth of a maximum (base 2) that rescales the accumulator
constexpr float kPaUp = 5.f;              // weights are at most 2^(kPaLazy + kPaUp): f16 keeps small ones exact
constexpr float kPaMost = 8192.f;         // 2^(kPaLazy + kPaUp)
constexpr float kPaUnset = -3e38f;        // the reference of a vector that has seen no key
constexpr float kPaLog2e = 1.4426950408889634f;

// A share's part of one group.
struct __align__(16) PaPiece {
  int len, row0, h, n_vec;          // the sequence's length and first row; KV head; vectors of the tile
  int row_lo, rest, row_hi, held_end;   // the tile's rows (and where in the first it begins); positions that are somebody's
  int s0, s1, cut, whole;           // its blocks; it begins inside the group; it is all of the group's blocks
  int g_begin, g_end, b, valid;     // units of the group's blocks (the share goes on at g_end); sequence
};
struct PaPlan {
  int S, n_teams, total, share_q, share_r, over;
};

template <int HD, int NT, bool PAIR>
struct PaShape {
  // sixteen warps where their registers allow it (128 a thread; two tiles of hd 128 spill
  // 128 bytes at that, an f32 tile of hd 128 48)
  static constexpr int kWarps = NT * (PAIR ? 2 : 1) <= 2 ? 16 : 8;
  static constexpr int kThreads = kWarps * 32;
  static constexpr int kTeams = kWarps / kPaTeam;            // most teams of a CTA
  static constexpr int kHalf = kPaKeys * HD;                 // K (or V) codes of a block
  static constexpr int kStage = 2 * kHalf;
  static constexpr int kStages = (HD == 128 ? 3 : 6) * (16 / kWarps) - (kWarps == 8 ? 1 : 0);
  static constexpr int kRing = kWarps * kStages * kStage;
  static constexpr int kQ = NT * HD * 16 * (PAIR ? 2 : 1);   // query fragments of a team
  static constexpr int kVec = NT * 8 * 12;                   // per vector: factor, then slope and position
  static constexpr int kQAt = kRing;
  static constexpr int kVecAt = kQAt + kTeams * kQ;
  static constexpr int kUnitsAt = kVecAt + kTeams * kVec;
  // a warp's partial result (8 NT rows of HD + 4 floats, a maximum and a sum each) lies in its ring
  static_assert(NT * 8 * (HD + 6) * 4 <= kStages * kStage, "partial results");
  static_assert(kTeams <= kPagedTeams, "the workspace");
  static_assert(kUnitsAt + 8 * (kPagedMaxSeqs + 1) + 1536 <= 232448, "shared memory");
};

__device__ __forceinline__ float pa_ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float pa_lg2(float x) {
  float y;
  asm("lg2.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, uint32_t n) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
}
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, uint64_t policy) {
  asm volatile("cp.async.cg.shared.global.L2::cache_hint [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "l"(policy)
               : "memory");
}
__device__ __forceinline__ void prefetch_l2(const void* p) { asm volatile("prefetch.global.L2 [%0];" ::"l"(p)); }
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void cp_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
__device__ __forceinline__ uint4 lds16(uint32_t a) {
  uint4 v;
  asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ uint2 lds8(uint32_t a) {
  uint2 v;
  asm volatile("ld.shared.v2.b32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ void mma_f16_16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                              uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t movmatrix_trans(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ uint32_t pack_f16x2(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ void split_f16x2(float a, float b, uint32_t& hi, uint32_t& lo) {
  const __half2 h = __floats2half2_rn(a, b);
  const float2 f = __half22float2(h);
  hi = *reinterpret_cast<const uint32_t*>(&h);
  lo = pack_f16x2(a - f.x, b - f.y);
}
__device__ __forceinline__ uint32_t hsub2_1152(uint32_t x) {
  const uint32_t c = 0x64806480u;   // 1152, 1152
  const __half2 r = __hsub2(*reinterpret_cast<const __half2*>(&x), *reinterpret_cast<const __half2*>(&c));
  return *reinterpret_cast<const uint32_t*>(&r);
}
// Codes 0, 1 and 2, 3 of a word as two f16 pairs.  int8: the byte with its sign
// bit turned is code + 128, and 0x6400 | byte is the f16 number 1024 + byte.
template <bool E4M3>
__device__ __forceinline__ void codes_f16(uint32_t w, uint32_t& a, uint32_t& b) {
  if (E4M3) {
    e4m3x4_to_f16(w, a, b);
  } else {
    const uint32_t u = w ^ 0x80808080u;
    a = hsub2_1152(__byte_perm(u, 0x64646464u, 0x4140));
    b = hsub2_1152(__byte_perm(u, 0x64646464u, 0x4342));
  }
}

// Byte offset of 16-byte chunk `ch` of row `r` (0..31) in a block's K or V
// codes.  Chunks are permuted so that the fragment loads of both products
// (8 lanes: two rows by four chunks, or four rows two apart by two chunks)
// and the row-wise copies meet no bank twice.
template <int HD>
__device__ __forceinline__ uint32_t pa_chunk(int r, int ch) {
  if (HD == 128) return r * 128u + ((ch ^ ((((r ^ (r >> 2)) & 1) << 2) | (r & 2))) << 4);
  return (r >> 1) * 128u + (((r ^ (r >> 1)) & 1) << 6) + ((ch ^ (((r >> 2) & 1) << 1)) << 4);
}

}  // namespace

template <bool E4M3, int HD, int NT, bool PAIR, bool FINE>
__global__ void __launch_bounds__(PaShape<HD, NT, PAIR>::kThreads, 1)
    paged_attend_kernel(const __grid_constant__ PagedAttendArgs a) {
  using SH = PaShape<HD, NT, PAIR>;
  constexpr int NV = 8 * NT;                 // vectors per tile
  constexpr int kSteps = HD / 16;            // k-steps of the scores, and 16-dim tiles of the output
  constexpr int kParts = PAIR ? 2 : 1;
  constexpr int W = SH::kWarps, ST = SH::kStages;
  extern __shared__ __align__(128) uint8_t sm[];
  const PagedArgs& c = a.c;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
  uint8_t* ring = sm + warp * ST * SH::kStage;
  const uint32_t ring_s = smem_u32(ring);
  int2* before = reinterpret_cast<int2*>(sm + SH::kUnitsAt);      // [n_seqs + 1] blocks, groups before a sequence
  constexpr int kFew = 32;                                        // sequences whose numbers one warp holds
  __shared__ PagedSeq few_s[kFew];
  __shared__ PaPiece piece_s[SH::kTeams][2];
  __shared__ PaPlan plan_s;
  __shared__ int2 scan_s[W];
  __shared__ int last_s[SH::kTeams];
  __shared__ int2 teams_s[SH::kTeams];
  const int G = a.G;

  if (!a.beside) griddep_wait();
  griddep_launch();
  {
    // what the pieces will ask for first, on its way to L2 while one warp plans: a
    // line of the page table and one of the queries for each thread of the grid
    const size_t i = static_cast<size_t>(blockIdx.x) * SH::kThreads + tid;
    const size_t table_bytes = static_cast<size_t>(c.n_seqs) * c.max_pages * 4;
    const size_t q_bytes = (static_cast<size_t>(c.n_rows - 1) * a.ld_q + a.n_heads * HD) * (a.dtype == DVI_BF16 ? 2 : 4);
    if (warp > 0 && i * 128 < table_bytes) prefetch_l2(reinterpret_cast<const uint8_t*>(c.table) + i * 128);
    if (warp > 0 && i * 128 < q_bytes) prefetch_l2(static_cast<const uint8_t*>(a.q) + i * 128);
  }

  // ---------------- sequences
  // Blocks [first, first + n) of a sequence that any of its rows sees, its tiles.
  auto extent = [&](int len, int rows, int& first, int& tiles) {
    const int vecs = rows * G;                              // the host refuses more than 2^31
    first = tiles = 0;
    if (rows <= 0 || vecs < a.min_vectors || vecs > a.max_vectors) return 0;
    const int end = min(len + rows, c.max_pages << c.log_p);
    if (a.window > 0) first = max(0, len - a.window + 1) / kPaKeys;
    tiles = static_cast<int>((static_cast<unsigned>(vecs) + NV - 1) / NV);
    return max(1, (end + kPaKeys - 1) / kPaKeys - first);   // at least one, so that empty rows are written
  };
  auto find = [&](int u, int u_end) {
    PaPiece r;
    r.valid = 0;
    if (u >= u_end) return r;
    const int over = plan_s.over;
    int b = 0;
    for (int hi = c.n_seqs - 1; b < hi;) {                  // the last b whose units begin at or before u
      const int mid = (b + hi + 1) >> 1;
      if (before[mid].x + before[mid].y * over <= u) b = mid;
      else hi = mid - 1;
    }
    const PagedSeq sq = c.n_seqs <= kFew ? few_s[b] : paged_seq(c, b);
    int first, tiles;
    const int n_blocks = extent(sq.len, sq.n, first, tiles), unit0 = before[b].x + before[b].y * over;
    int grp = static_cast<int>(__fdividef(static_cast<float>(u - unit0), static_cast<float>(n_blocks + over)));
    while (grp * (n_blocks + over) > u - unit0) --grp;      // (u - unit0) / (n_blocks + over), exactly
    while ((grp + 1) * (n_blocks + over) <= u - unit0) ++grp;
    r.g_begin = unit0 + grp * (n_blocks + over) + over;
    r.g_end = r.g_begin + n_blocks;
    const int blk0 = max(u - r.g_begin, 0), blk1 = min(u_end, r.g_end) - r.g_begin;
    if (blk1 <= 0) return r;                                // the share ends before the group's first block
    const int tile = tiles == 1 ? 0 : grp % tiles;
    r.h = tiles == 1 ? grp : grp / tiles;
    const int n0 = tile * NV;                               // first vector
    r.n_vec = min(NV, sq.n * G - n0);
    r.row_lo = tile == 0 ? 0 : n0 / G;
    r.rest = n0 - r.row_lo * G;
    r.row_hi = r.row_lo + (G == 1 ? r.n_vec - 1 : static_cast<int>(__umulhi(static_cast<uint32_t>(r.rest + r.n_vec - 1), a.inv_g)));
    // positions that some row of the tile sees
    const int cap = c.max_pages << c.log_p;
    const int see_end = min(sq.len + r.row_hi + 1, cap);
    const int see_begin = a.window > 0 ? max(0, sq.len + r.row_lo - a.window + 1) : 0;
    r.held_end = min(sq.len + sq.n, cap);                   // rows of the cache past it are nobody's
    r.s0 = max(first + blk0, see_begin / kPaKeys);
    r.s1 = min(first + blk1, (see_end + kPaKeys - 1) / kPaKeys);
    r.len = sq.len;
    r.row0 = sq.row0;
    r.cut = blk0 > 0;
    r.whole = blk0 == 0 && blk1 == n_blocks;
    r.b = b;
    r.valid = 1;
    return r;
  };
  // floor(total k / n_teams); the fraction's numerator is below 2^20, so f32 decides it
  auto share = [&](int k) {
    return plan_s.share_q * k +
           static_cast<int>(__fdividef(static_cast<float>(plan_s.share_r * k) + 0.5f, static_cast<float>(plan_s.n_teams)));
  };
  int2 all = make_int2(0, 0);                                    // blocks and groups of all sequences
  for (int b0 = 0; b0 < c.n_seqs; b0 += SH::kThreads) {
    if (c.n_seqs <= kFew && warp > 0) break;
    const int b = b0 + tid;
    int n = 0, ng = 0;
    if (b < c.n_seqs) {
      int first, tiles;
      const PagedSeq sq = paged_seq(c, b);
      const int blocks = extent(sq.len, sq.n, first, tiles);
      ng = tiles * c.H;
      n = blocks * ng;
      if (c.n_seqs <= kFew) few_s[b] = sq;
    }
#pragma unroll 1
    for (int o = 1; o < min(c.n_seqs, 32); o <<= 1) {
      const int x = __shfl_up_sync(0xffffffffu, n, o), y = __shfl_up_sync(0xffffffffu, ng, o);
      if (lane >= o) n += x, ng += y;
    }
    if (c.n_seqs <= kFew) {
      if (b < c.n_seqs) before[b + 1] = make_int2(n, ng);
      const int last = c.n_seqs - 1;
      all = make_int2(__shfl_sync(0xffffffffu, n, last), __shfl_sync(0xffffffffu, ng, last));
    } else {
      if (b0 > 0) __syncthreads();
      if (lane == 31) scan_s[warp] = make_int2(n, ng);
      __syncthreads();
      int2 at = all;
#pragma unroll 4
      for (int w = 0; w < W; ++w) {
        const int2 x = scan_s[w];
        if (w < warp) at.x += x.x, at.y += x.y;
        all.x += x.x, all.y += x.y;
      }
      if (b < c.n_seqs) before[b + 1] = make_int2(at.x + n, at.y + ng);
    }
  }
  if (tid == 0) before[0] = make_int2(0, 0);
  if (c.n_seqs > kFew) __syncthreads();

  // ---------------- plan (one warp): teams of S warps take equal shares of a row of
  // units, a group's being as many as its blocks and `over` = S more for what a
  // group costs beside them (a step of each warp).  Groups of equal size are not
  // cut across a share where each share holds one part.  16 warps on a group while
  // that leaves each of them two steps (32 where a share holds several groups: the
  // small teams of an SM work through one group's start and end beside another's
  // blocks) and the shares fill the GPU nearly as well as smaller teams' would.
  if (warp == 0) {
    const int groups = all.y;
    // lane e weighs teams of W >> e warps
    int n_teams = 0;
    float fill = -1.f;
    {
      const int log = 31 - __clz(W) - min(lane, 2), s = 1 << log, most = static_cast<int>(gridDim.x) * (W >> log);
      if (s == kPaTeam || all.x >= (groups > most ? 32 : 2) * s * groups) {
        // a share is two steps at least, but no group waits for another while a team is free
        const int few = max(groups, (all.x + groups * s) >> (log + 1));
        n_teams = min(most, few);
        fill = 0.9f;
        if (n_teams >= groups) {
          int k = static_cast<int>(__fdividef(static_cast<float>(n_teams), static_cast<float>(max(groups, 1))));
          k += (k + 1) * groups <= n_teams ? 1 : 0;                      // n_teams / groups, exactly
          k -= k * groups > n_teams ? 1 : 0;
          n_teams = k * groups;
          fill = __fdividef(static_cast<float>(n_teams), static_cast<float>(most));
        }
      }
    }
    int pick = 0;
    float best = __shfl_sync(0xffffffffu, fill, 0);
#pragma unroll
    for (int e = 1; (W >> e) >= kPaTeam; ++e) {
      const float f = __shfl_sync(0xffffffffu, fill, e);
      if (best < 0.f || f > best + 0.2f) best = f, pick = e;
    }
    const int S = W >> pick;
    n_teams = __shfl_sync(0xffffffffu, n_teams, pick);
    const int total = all.x + groups * S * kPaOver;
    if (lane == 0) {
      plan_s.S = S, plan_s.over = S * kPaOver;
      plan_s.n_teams = n_teams, plan_s.total = total;
      plan_s.share_q = n_teams > 0 ? total / n_teams : 0;
      plan_s.share_r = total - plan_s.share_q * n_teams;
    }
    __syncwarp();
    if (lane < W / S) {
      const int team = lane * static_cast<int>(gridDim.x) + static_cast<int>(blockIdx.x);
      if (team < n_teams) piece_s[lane][0] = find(share(team), share(team + 1));
      else piece_s[lane][0].valid = 0;
    }
  }
  __syncthreads();
  const int S = plan_s.S, log_s = 31 - __clz(S);
  const int tw = warp & (S - 1), in_cta = warp >> log_s;
  const int team = in_cta * static_cast<int>(gridDim.x) + static_cast<int>(blockIdx.x);
  auto team_of = [&](int unit) {
    const int n_teams = plan_s.n_teams;
    int k = min(n_teams - 1, static_cast<int>(static_cast<float>(unit) *
                                              (static_cast<float>(n_teams) / static_cast<float>(plan_s.total))));
    while (k > 0 && share(k) > unit) --k;
    while (share(k + 1) <= unit) ++k;
    return k;
  };
  auto team_bar = [&] { named_bar(1 + in_cta, 32 * S); };
  const uint64_t once = l2_evict_first_policy();   // codes are read once; tables, queries and parts are to stay
  uint8_t* qf = sm + SH::kQAt + in_cta * SH::kQ;
  const uint32_t q_s = smem_u32(qf);
  float* fac = reinterpret_cast<float*>(sm + SH::kVecAt + in_cta * SH::kVec);
  float2* vec = reinterpret_cast<float2*>(fac + NV);

  for (int turn = 0;; turn ^= 1) {
    const PaPiece pc = piece_s[in_cta][turn];
    if (!pc.valid) break;
    const int len = pc.len, h = pc.h, n_vec = pc.n_vec, s0 = pc.s0, s1 = pc.s1, held_end = pc.held_end;
    auto row_of = [&](int n, int& hq) {                            // vector n of the tile: its row, its head
      const int r = G == 1 ? n : static_cast<int>(__umulhi(static_cast<uint32_t>(pc.rest + n), a.inv_g));
      hq = h * G + pc.rest + n - r * G;
      return pc.row_lo + r;
    };

    // ---------------- the warp's blocks s0 + tw + i S.  Lane i % 32 holds the table
    // entry of block i, and its page's scales: entries are read 32 blocks ahead
    const int n_mine = s1 - s0 - tw > 0 ? (s1 - s0 - tw + S - 1) >> log_s : 0;
    auto entry = [&](int i) {
      return i < n_mine ? paged_entry(c, pc.b, ((s0 + tw + (i << log_s)) * kPaKeys) >> c.log_p) : -1;
    };
    int ent = entry(lane), ent_next = -1;

    // ---------------- queries: a warp loads whole vectors, HD / 32 dims a lane, as they lie there
    constexpr int kDims = HD / 32;
    constexpr int kMine = NV / kPaTeam;                            // most vectors of a warp
    uint32_t qx[kMine][PAIR ? kDims : kDims / 2];
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
      const int n = tw + i * S;
#pragma unroll
      for (int e = 0; e < (PAIR ? kDims : kDims / 2); ++e) qx[i][e] = 0u;
      if (n < n_vec) {
        int hq;
        const int row = row_of(n, hq);
        const uint32_t* p = static_cast<const uint32_t*>(a.q) +
                            (static_cast<long long>(pc.row0 + row) * a.ld_q + hq * HD + lane * kDims) / (PAIR ? 1 : 2);
#pragma unroll
        for (int e = 0; e < (PAIR ? kDims : kDims / 2); ++e) qx[i][e] = p[e];
      }
    }

    // ---------------- copies
    const float* ks_h = c.k_scale + h;
    const float* vs_h = c.v_scale + h;
    constexpr int kRow = HD / 16;                                  // 16-byte chunks of a row
    constexpr int kRows = 32 / kRow;                               // rows a warp copies at once
    const int r0 = lane / kRow, ch = lane % kRow;
    const size_t page_bytes = (static_cast<size_t>(c.H) << c.log_p) * HD;
    const uint8_t* k_lane = c.k + ((static_cast<size_t>(h) << c.log_p) + r0) * HD + ch * 16;
    const long long v_from_k = c.v - c.k;
    // the permutation has a period of 8 rows: at most two lane offsets
    const uint32_t at0 = ring_s + pa_chunk<HD>(r0, ch), at1 = ring_s + pa_chunk<HD>(r0 + kRows, ch);
    auto copy = [&](int i, int stage) {
      const int pg = __shfl_sync(0xffffffffu, ent, i & 31);
      const int p = (s0 + tw + (i << log_s)) * kPaKeys;
      const uint8_t* src = k_lane + static_cast<size_t>(max(pg, 0)) * page_bytes + (p & (c.P - 1)) * HD;
      const uint32_t d0 = at0 + stage * SH::kStage, d1 = at1 + stage * SH::kStage;
      if (pg >= 0 && p + kPaKeys <= held_end) {
#pragma unroll
        for (int r = 0; r < kPaKeys / kRows; ++r) {
          const uint32_t dst = (r & 1 ? d1 : d0) + (r >> 1) * 2 * kRows * HD;
          cp_async16(dst, src + r * kRows * HD, once);
          cp_async16(dst + SH::kHalf, src + v_from_k + r * kRows * HD, once);
        }
      } else {
        const int live = pg >= 0 ? held_end - p - r0 : 0;          // rows past it, and pages not held: zeros
#pragma unroll 1
        for (int r = 0; r < kPaKeys / kRows; ++r) {
          const uint32_t n = r * kRows < live ? 16u : 0u;
          const uint32_t dst = (r & 1 ? d1 : d0) + (r >> 1) * 2 * kRows * HD;
          cp_async16(dst, src + r * kRows * HD, n);
          cp_async16(dst + SH::kHalf, src + v_from_k + r * kRows * HD, n);
        }
      }
    };

    float ks_in, vs_in;                          // scales of the blocks being copied
    auto batch = [&](int j) {                    // block j is the first of 32
      ent = paged_valid(c, ent);
      ent_next = entry(j + 32 + lane);
      ks_in = ent >= 0 ? __ldg(ks_h + static_cast<size_t>(ent) * c.H) : 0.f;
      vs_in = ent >= 0 ? __ldg(vs_h + static_cast<size_t>(ent) * c.H) : 0.f;
    };
    batch(0);
#pragma unroll 1
    for (int j = 0; j < ST - 1; ++j) {
      if (j < n_mine) copy(j, j);
      cp_commit();
    }
    if (tw == S - 1 && lane == 0) {
      // (teams of the group, for the join: this warp has time)
      if (!pc.whole) teams_s[in_cta] = make_int2(team_of(pc.g_begin), team_of(pc.g_end - 1));
      piece_s[in_cta][turn ^ 1] = find(pc.g_end, share(team + 1));
    }

    // ---------------- query fragments: thread (g, t) of vector 8 nt + g holds, for
    // step j, dims 16 t + 4 j .. + 3 (hd 128: from step 4 on 64 + 16 t + 4 (j - 4))
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
      const int n = tw + i * S;
      if (n >= NV) continue;
      float x[kDims];
#pragma unroll
      for (int e = 0; e < kDims; ++e)
        x[e] = PAIR ? __uint_as_float(qx[i][PAIR ? e : 0]) : e & 1 ? bf16_hi(qx[i][e >> 1]) : bf16_lo(qx[i][e >> 1]);
      float top = 0.f;
#pragma unroll
      for (int e = 0; e < kDims; ++e) top = fmaxf(top, fabsf(x[e]));
      top = warp_max(top);
      // a power of two brings the largest element to [2^14, 2^15)
      const int ex = max(static_cast<int>(__float_as_uint(top) >> 23), 15);
      const float up = __uint_as_float(static_cast<uint32_t>(268 - ex) << 23);
      const float down = __uint_as_float(static_cast<uint32_t>(ex - 14) << 23);
      const int d = lane * kDims;
      uint8_t* at = qf + (((n >> 3) * kSteps + (d / 64) * 4 + (d % 16) / 4) * 32 + (n & 7) * 4 + (d % 64) / 16) * 8 +
                    (d % 4) * 2;
#pragma unroll
      for (int e = 0; e < kDims; e += 2) {
        uint32_t hi, lo;
        split_f16x2(x[e] * up, x[e + 1] * up, hi, lo);
        *reinterpret_cast<uint32_t*>(at + e * 2) = hi;
        if (PAIR) *reinterpret_cast<uint32_t*>(at + NT * kSteps * 256 + e * 2) = lo;
      }
      if (lane == 0) {
        int hq;
        const int row = row_of(n, hq);
        const bool live = n < n_vec;
        const float f = !FINE && a.softcap > 0.f ? down * (a.scale / a.softcap) : down * (a.scale * kPaLog2e);
        fac[n] = f;
        vec[n] = make_float2(live && a.slopes ? __ldg(a.slopes + hq) * kPaLog2e : 0.f,
                             __int_as_float(live ? len + row : -1));
      }
    }
    team_bar();

    float o[kSteps][NT][4];
    float m[NT][2], l[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
      for (int i = 0; i < kSteps; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[i][nt][e] = 0.f;
      m[nt][0] = m[nt][1] = kPaUnset;
      l[nt][0] = l[nt][1] = 0.f;
    }

    // blocks that every row of the tile sees whole: full_begin .. full_end - 1
    const int full_end = min((len + pc.row_lo + 1) / kPaKeys, held_end / kPaKeys);
    const int full_begin = a.window > 0 ? max(0, len + pc.row_hi - a.window + kPaKeys) / kPaKeys : 0;
    const bool curved = FINE || a.softcap > 0.f || a.slopes != nullptr;
    float ks_l = 0.f, lv_l = 0.f, iv_l = 0.f;    // ks, log2 vs and 1 / vs (0: no page) of the blocks at work
    int stage = 0;
#pragma unroll 1
    for (int i = 0; i < n_mine; ++i) {
      if ((i & 31) == 0) {
        const float x = fmaxf(vs_in, kPagedMinScale);
        ks_l = ks_in, lv_l = pa_lg2(x), iv_l = vs_in > 0.f ? __fdividef(1.f, x) : 0.f;
      }
      {
        const int j = i + ST - 1;                // its copies go where the last step read
        if (j < n_mine) {
          if ((j & 31) == 0) {
            ent = ent_next;
            batch(j);
          }
          __syncwarp();
          copy(j, stage == 0 ? ST - 1 : stage - 1);
        }
        cp_commit();
      }
      cp_wait<ST - 1>();
      __syncwarp();
      const int blk = s0 + tw + (i << log_s);
      const float ks = __shfl_sync(0xffffffffu, ks_l, i & 31), iv = __shfl_sync(0xffffffffu, iv_l, i & 31);
      float lv = __shfl_sync(0xffffffffu, lv_l, i & 31);
      const uint32_t ks_s = ring_s + stage * SH::kStage, vs_s = ks_s + SH::kHalf;
      // ---------------- scores
      float s[NT][4];
      {
        uint32_t w0[kSteps], w1[kSteps];   // codes of keys g and g + 8
#pragma unroll
        for (int i = 0; i < HD / 64; ++i) {
          const uint4 x = lds16(ks_s + pa_chunk<HD>(g, 4 * i + t));
          const uint4 y = lds16(ks_s + pa_chunk<HD>(g + 8, 4 * i + t));
          w0[4 * i] = x.x, w0[4 * i + 1] = x.y, w0[4 * i + 2] = x.z, w0[4 * i + 3] = x.w;
          w1[4 * i] = y.x, w1[4 * i + 1] = y.y, w1[4 * i + 2] = y.z, w1[4 * i + 3] = y.w;
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int e = 0; e < 4; ++e) s[nt][e] = 0.f;
#pragma unroll
        for (int j = 0; j < kSteps; ++j) {
          uint32_t a0, a1, a2, a3;
          codes_f16<E4M3>(w0[j], a0, a2);
          codes_f16<E4M3>(w1[j], a1, a3);
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int part = 0; part < kParts; ++part) {
              const uint2 q = lds8(q_s + ((part * NT + nt) * kSteps + j) * 256 + lane * 8);
              mma_f16_16816(s[nt], a0, a1, a2, a3, q.x, q.y);
            }
        }
      }
      // ---------------- softmax: element e of s[nt]: key g + 8 (e / 2), vector 8 nt + 2 t + e % 2
      const bool plain = blk >= full_begin && blk < full_end && iv > 0.f;
      float f[NT][2];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        const float2 x = *reinterpret_cast<const float2*>(fac + nt * 8 + 2 * t);
        f[nt][0] = x.x * ks, f[nt][1] = x.y * ks;
      }
      if (!plain || curved) {
        // the finished scores in place of the products
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          const float4 v = *reinterpret_cast<const float4*>(vec + nt * 8 + 2 * t);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            float x = s[nt][e] * f[nt][e & 1];
            if (FINE) {
              x = paged_cap_fine(x, a.cap);
            } else if (a.softcap > 0.f) {
              if (PAIR) x = tanhf(x);
              else x = 1.f - __fdividef(2.f, 1.f + pa_ex2(x * (2.f * kPaLog2e)));
              x *= a.softcap * kPaLog2e;
            }
            const int d = blk * kPaKeys + g + 8 * (e >> 1) - __float_as_int(e & 1 ? v.w : v.y);
            x = fmaf(e & 1 ? v.z : v.x, static_cast<float>(d), x + lv);
            if (!plain && (d > 0 || !(iv > 0.f) || (a.window > 0 && d <= -a.window))) x = -INFINITY;
            s[nt][e] = x;
          }
          f[nt][0] = f[nt][1] = 1.f;
        }
        lv = 0.f;
      }
      float p[NT][4], most = 0.f;
      auto weights = [&] {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          // (the score is rounded as it is for the maximum, before the reference goes off:
          // one multiply-add for both would leave the rounding of a huge score in the exponent)
#pragma unroll
          for (int e = 0; e < 4; ++e) p[nt][e] = pa_ex2(fmaf(s[nt][e], f[nt][e & 1], lv) - m[nt][e & 1]);
        }
      };
      weights();
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 4; ++e) most = fmaxf(most, p[nt][e]);
      if (__any_sync(0xffffffffu, most > kPaMost)) {
        // some maximum has outgrown its reference (or is the first)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int q = 0; q < 2; ++q) {
            float x = fmaxf(fmaf(s[nt][q], f[nt][q], lv), fmaf(s[nt][q + 2], f[nt][q], lv));
#pragma unroll
            for (int off = 4; off < 32; off <<= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, off));
            x = fmaxf(x - kPaUp, m[nt][q]);                       // the reference sits below the maximum
            const float shrink = pa_ex2(m[nt][q] - x);
            m[nt][q] = x;
            l[nt][q] *= shrink;
#pragma unroll
            for (int i = 0; i < kSteps; ++i) o[i][nt][q] *= shrink, o[i][nt][q + 2] *= shrink;
          }
        weights();
      }
      uint32_t pb[NT][2], pl[NT][2];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        l[nt][0] = fmaf(p[nt][0] + p[nt][2], iv, l[nt][0]);
        l[nt][1] = fmaf(p[nt][1] + p[nt][3], iv, l[nt][1]);
        if (PAIR) {
          uint32_t h0, h1, l0, l1;
          split_f16x2(p[nt][0], p[nt][1], h0, l0);
          split_f16x2(p[nt][2], p[nt][3], h1, l1);
          pb[nt][0] = movmatrix_trans(h0), pb[nt][1] = movmatrix_trans(h1);
          pl[nt][0] = movmatrix_trans(l0), pl[nt][1] = movmatrix_trans(l1);
        } else {
          pb[nt][0] = movmatrix_trans(pack_f16x2(p[nt][0], p[nt][1]));
          pb[nt][1] = movmatrix_trans(pack_f16x2(p[nt][2], p[nt][3]));
        }
      }
      // ---------------- values: keys 2 t, 2 t + 1, 2 t + 8, 2 t + 9, HD / 8 dims from g HD / 8 on
      {
        constexpr int kW = HD / 32;                                // words of a thread's dims
        uint32_t w[4][kW];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int r = 2 * t + (k & 1) + 8 * (k >> 1);
          if (HD == 128) {
            const uint4 x = lds16(vs_s + pa_chunk<HD>(r, g));
            w[k][0] = x.x, w[k][1] = x.y, w[k][kW - 2] = x.z, w[k][kW - 1] = x.w;
          } else {
            const uint2 x = lds8(vs_s + pa_chunk<HD>(r, g >> 1) + (g & 1) * 8);
            w[k][0] = x.x, w[k][1] = x.y;
          }
        }
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
          const uint32_t sel = i & 1 ? 0x7362u : 0x5140u;          // dims 2 i and 2 i + 1 of two keys
          uint32_t a0, a1, a2, a3;
          codes_f16<E4M3>(__byte_perm(w[0][i >> 1], w[1][i >> 1], sel), a0, a1);
          codes_f16<E4M3>(__byte_perm(w[2][i >> 1], w[3][i >> 1], sel), a2, a3);
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            if (PAIR) {
              // a fresh accumulator each step: the sum over thousands of steps rounds to nearest
              float d[4] = {0.f, 0.f, 0.f, 0.f};
              mma_f16_16816(d, a0, a1, a2, a3, pl[nt][0], pl[nt][1]);
              mma_f16_16816(d, a0, a1, a2, a3, pb[nt][0], pb[nt][1]);
#pragma unroll
              for (int e = 0; e < 4; ++e) o[i][nt][e] += d[e];
            } else {
              mma_f16_16816(o[i][nt], a0, a1, a2, a3, pb[nt][0], pb[nt][1]);
            }
          }
        }
      }
      stage = stage + 1 == ST ? 0 : stage + 1;
    }
    cp_wait<0>();
    __syncwarp();

    // ---------------- join.  o[i][nt][e] is dim g HD/8 + 2 i + e / 2 of vector 8 nt + 2 t + e % 2; a warp's
    // part lies in its ring as rows of [i][g] pairs, 4 floats apart from HD so that no bank meets twice
    constexpr int kPart = HD + 4;
    float* mine = reinterpret_cast<float*>(ring);                  // [NV][kPart], maxima [NV], sums [NV]
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        float x = l[nt][q];
#pragma unroll
        for (int off = 4; off < 32; off <<= 1) x += __shfl_xor_sync(0xffffffffu, x, off);
        const int n = nt * 8 + 2 * t + q;
        if (g == 0) {
          mine[NV * kPart + n] = m[nt][q];
          mine[NV * kPart + NV + n] = x;
        }
#pragma unroll
        for (int i = 0; i < kSteps; ++i)
          *reinterpret_cast<float2*>(mine + n * kPart + i * 16 + g * 2) = make_float2(o[i][nt][q], o[i][nt][q + 2]);
      }
    team_bar();
    const bool whole = pc.whole;
    // a part in the workspace: [NV][HD / 4] quads as they lie here, maxima [NV], sums [NV]
    constexpr int kSlot = NV * (HD + 2);
    const int quads = n_vec * (HD / 4);
    float* slot = a.part + static_cast<size_t>(2 * team + (pc.cut ? 0 : 1)) * kSlot;
    auto emit = [&](int i, float4 acc, float L) {                  // quad i: dims d, d + 1 and d + HD / 8, d + HD / 8 + 1
      const int v = i / (HD / 4), d = (i % 4) * (HD / 4) + i % (HD / 4) / 4 * 2;
      const float inv = L > 0.f ? __fdividef(1.f, L) : (L == L ? 0.f : L);
      int hq;
      const int row = row_of(v, hq);
      const long long off = static_cast<long long>(pc.row0 + row) * a.ld_o + hq * HD + d;
      if (PAIR) {
        float* at = static_cast<float*>(a.o) + off;
        *reinterpret_cast<float2*>(at) = make_float2(acc.x * inv, acc.y * inv);
        *reinterpret_cast<float2*>(at + HD / 8) = make_float2(acc.z * inv, acc.w * inv);
      } else {
        __nv_bfloat16* at = static_cast<__nv_bfloat16*>(a.o) + off;
        *reinterpret_cast<uint32_t*>(at) = pack_bf16x2(acc.x * inv, acc.y * inv);
        *reinterpret_cast<uint32_t*>(at + HD / 8) = pack_bf16x2(acc.z * inv, acc.w * inv);
      }
    };
    constexpr int kWarpFloats = ST * SH::kStage / 4;
    const float* parts = reinterpret_cast<const float*>(sm) + in_cta * S * kWarpFloats;
#pragma unroll 1
    for (int i = tw * 32 + lane; i < quads; i += S * 32) {
      const int v = i / (HD / 4);
      const float* head = parts + NV * kPart + v;
      const float* quad = parts + v * kPart + i % (HD / 4) * 4;
      float M = kPaUnset, L = 0.f;
#pragma unroll 8
      for (int w = 0; w < S; ++w) M = fmaxf(M, head[w * kWarpFloats]);
      float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
      for (int w = 0; w < S; ++w) {
        const float f = pa_ex2(head[w * kWarpFloats] - M);
        const float4 x = *reinterpret_cast<const float4*>(quad + w * kWarpFloats);
        acc.x = fmaf(x.x, f, acc.x), acc.y = fmaf(x.y, f, acc.y);
        acc.z = fmaf(x.z, f, acc.z), acc.w = fmaf(x.w, f, acc.w);
        L = fmaf(head[w * kWarpFloats + NV], f, L);
      }
      if (whole) {
        emit(i, acc, L);
      } else {
        __stcg(reinterpret_cast<float4*>(slot) + i, acc);
        if (i % (HD / 4) == 0) {
          __stcg(slot + NV * HD + v, M);
          __stcg(slot + NV * HD + NV + v, L);
        }
      }
    }
    if (!whole) {
      // teams of the group: t0 .. t1; whoever of them counts last joins their parts in order
      const int t0 = teams_s[in_cta].x, t1 = teams_s[in_cta].y;
      team_bar();
      if (tw == 0 && lane == 0) {
        const int n = paged_arrive(a.counters + t0);
        last_s[in_cta] = n == t1 - t0;
        if (n == t1 - t0) a.counters[t0] = 0;
      }
      team_bar();
      if (last_s[in_cta]) {
        const float* p0 = a.part + static_cast<size_t>(2 * t0 + 1) * kSlot;
        const float* p1 = a.part + static_cast<size_t>(2 * t0) * kSlot;
        const int n = t1 - t0 + 1;
#pragma unroll 1
        for (int i = tw * 32 + lane; i < quads; i += S * 32) {
          const int v = i / (HD / 4);
          float M = kPaUnset, L = 0.f;
          float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
          constexpr int kAtOnce = 6;
#pragma unroll 1
          for (int k0 = 0; k0 < n; k0 += kAtOnce) {
            float pm[kAtOnce], ps[kAtOnce];
            float4 x[kAtOnce];
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k) {
              const float* p = k0 + k == 0 ? p0 : p1 + static_cast<size_t>(2 * min(k0 + k, n - 1)) * kSlot;
              pm[k] = __ldcg(p + NV * HD + v), ps[k] = __ldcg(p + NV * HD + NV + v);
              x[k] = __ldcg(reinterpret_cast<const float4*>(p) + i);
            }
            float top = M;
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k) {
              if (k0 + k >= n) pm[k] = -INFINITY;
              top = fmaxf(top, pm[k]);
            }
            const float shrink = pa_ex2(M - top);
            M = top;
            acc.x *= shrink, acc.y *= shrink, acc.z *= shrink, acc.w *= shrink, L *= shrink;
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k) {
              const float f = pa_ex2(pm[k] - top);
              if (k0 + k < n) {
                acc.x = fmaf(x[k].x, f, acc.x), acc.y = fmaf(x[k].y, f, acc.y);
                acc.z = fmaf(x[k].z, f, acc.z), acc.w = fmaf(x[k].w, f, acc.w);
                L = fmaf(ps[k], f, L);
              }
            }
          }
          emit(i, acc, L);
        }
      }
    }
    team_bar();   // the rings and the queries are read before the next group's
  }
  if (a.beside) griddep_wait();   // whoever waits for this grid waits for the one before it too
}

namespace {
template <bool E4M3, int HD, int NT, bool PAIR, bool FINE = false>
cudaError_t launch_pa(const PagedAttendArgs& a, int n_sms, cudaStream_t s) {
  using SH = PaShape<HD, NT, PAIR>;
  // the units of all groups are counted in 32 bits
  const long long vecs = static_cast<long long>(a.c.n_rows) * a.G, tiles = vecs / (8 * NT) + a.c.n_seqs;
  const long long blocks = ((static_cast<long long>(a.c.max_pages) << a.c.log_p) / kPaKeys + 16 * kPaOver + 1) * a.c.H;
  if (vecs > 0x7fffffffll || tiles * blocks > 0x7fffffffll) return cudaErrorInvalidConfiguration;
  static PerDevice attr;
  attr.once([] {
    cudaFuncSetAttribute(paged_attend_kernel<E4M3, HD, NT, PAIR, FINE>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                         SH::kUnitsAt + 8 * (kPagedMaxSeqs + 1));
  });
  return launch_pdl(paged_attend_kernel<E4M3, HD, NT, PAIR, FINE>, dim3(n_sms), dim3(SH::kThreads),
                    SH::kUnitsAt + 8 * (a.c.n_seqs + 1), s, a);
}
template <bool E4M3, int HD>
cudaError_t pa_tiles(const PagedAttendArgs& a, int n_sms, cudaStream_t s) {
  const long long vecs = std::min<long long>(static_cast<long long>(a.c.max_rows) * a.G, a.max_vectors);
  if (a.dtype == DVI_F32)
    return vecs <= 8 ? launch_pa<E4M3, HD, 1, true>(a, n_sms, s) : launch_pa<E4M3, HD, 2, true>(a, n_sms, s);
  // large caps have kernels of their own, as both caps in one take 1 to 4 % of every call with a usual
  // cap or a bias (6 rows of 32 sequences behind 16384 positions, a bias: 214 to 221 us), and one tile
  // for all counts (64 single tokens 44 us, 34 under a usual cap in a tile of 8)
  if (a.cap.near > 0.f) return launch_pa<E4M3, HD, 2, false, true>(a, n_sms, s);
  // (24 vectors of 32 sequences, 4000 positions, 8 KV heads of 128: 71.3 us in a tile of
  // 24, 78.0 in one of 32)
  if (vecs <= 8) return launch_pa<E4M3, HD, 1, false>(a, n_sms, s);
  if (vecs <= 16) return launch_pa<E4M3, HD, 2, false>(a, n_sms, s);
  if (vecs <= 24) return launch_pa<E4M3, HD, 3, false>(a, n_sms, s);
  return launch_pa<E4M3, HD, 4, false>(a, n_sms, s);
}
}  // namespace

template <bool E4M3>
cudaError_t launch_paged_attend(const PagedAttendArgs& a, int n_sms, cudaStream_t s) {
  return a.c.D == 128 ? pa_tiles<E4M3, 128>(a, n_sms, s) : pa_tiles<E4M3, 64>(a, n_sms, s);
}

}  // namespace dvi
