// Token probabilities with cuts: w of a token as a whole number, whose sums do not depend on their order.
#pragma once

#include "token_probs.cuh"

namespace dvi {
namespace {

// Numbers T_k near 2^(k / kPowers) that are f32 numbers themselves, and how far log2 T_k is from
// k / kPowers: so 2^t = T_k 2^(t - k / kPowers - d_k) without a second number for T_k.
constexpr int kPowers = 1024;
struct Powers {
  float2 of[kPowers];
};
// e^x and the logarithm of numbers near 1 by their series, in 64 bits.
constexpr double series_exp(double x) {
  double sum = 1.0, term = 1.0;
  for (int i = 1; i < 30; ++i) sum += term *= x / i;
  return sum;
}
constexpr double series_log1p(double x) {
  double sum = 0.0, term = 1.0;
  for (int i = 1; i < 6; ++i) sum += (term *= x) / (i % 2 ? i : -i);
  return sum;
}
constexpr Powers make_powers() {
  constexpr double ln2 = 0.69314718055994530942;
  Powers p{};
  for (int k = 0; k < kPowers; ++k) {
    const double t = series_exp(k * (ln2 / kPowers));
    p.of[k].x = static_cast<float>(t);
    p.of[k].y = static_cast<float>(series_log1p((static_cast<double>(p.of[k].x) - t) / t) / ln2);
  }
  return p;
}
__device__ const Powers kPowersOf2 = make_powers();

// w in units of 2^-44, off by less than 2^-31 of itself; 0 below 2^-46 (low: where that is, or above).
// t = (x - m) c is x c less m c.  Adding 1.5 * 2^23 / kPowers rounds x c to multiples q of 1 / kPowers and
// leaves them in the low bits; the rest x c - q is one number, as a fused multiply-add rounds only what is
// left.  (|x c| stays below 4096: where |m c| does not, what counts is so near to m that x - m is exact and
// takes x's place.)  The rest of m c is in the table, turned by m's own q: 2^q from the table and an
// exponent, 2^u - 1 = u ln 2 + ... is small enough for one number.  w in 22 bits, then 22 more.
// What it is off by: u, below 3 2^-11, is rounded in six places, by 6 2^-35 together, 4.2 2^-35 of w; the cubic's
// coefficient and two roundings are 2.3 2^-24 of 2^u - 1 < 2^-9.9, 4.6 2^-35: 2^-31.8 if all went one way (found among
// 70 million: 2^-32.97, in the mean of a row 2^-35.6).  That is chosen: u and 2^u - 1 as two numbers each would take
// more instructions in the sums that many rows are bound by.
// Two numbers are weighed together: an operation on a register pair is one instruction.
struct Two {
  unsigned long long v;
};
__device__ __forceinline__ Two two(float a, float b) {
  Two r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ Two two(float a) { return two(a, a); }
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
__device__ __forceinline__ Two operator*(Two a, Two b) {
  Two r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
  return r;
}
__device__ __forceinline__ Two fma(Two a, Two b, Two c) {
  Two r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
  return r;
}
__device__ __forceinline__ Two operator-(Two a, Two b) { return fma(b, two(-1.f), a); }   // (the product is exact)

struct Weigher {
  float m;
  Slope c;
  const float2* powers;   // turned: by the low bits of the sum with kGrid, as bits that want (q's other bits) << 13 only
  float base;             // 0, or m
  float least;            // of x - base: w there is 2^-46, which rounds to 0, as it is below
  static constexpr float kGrid = 12582912.f / kPowers;
  // The two halves of each, beside kBits.
  static constexpr unsigned kBits = 0x4b400000u;   // of 1.5 * 2^23
  __device__ __forceinline__ Weigher(float m, Slope c, const float2* powers)
      : m(m), c(c), powers(powers), base(fabsf(m * c.hi) < 4000.f ? 0.f : m), least((m - base) - 46.f / c.hi * 1.0001f) {}
  __device__ __forceinline__ void halves(float x0, float x1, unsigned (&high)[2], unsigned (&rest)[2]) const {
    halves_by([of = powers](unsigned i) { return of[i]; }, x0, x1, high, rest);
  }
  template <typename F>
  __device__ __forceinline__ void halves_by(F power, float x0, float x1, unsigned (&high)[2], unsigned (&rest)[2]) const {
    const float2 xs = split(two(x0, x1) + two(-base));
    const Two kRound = two(12582912.f), ch = two(c.hi), x = two(fmaxf(xs.x, least), fmaxf(xs.y, least));
    const Two q = fma(x, ch, two(kGrid));
    const Two r = fma(x, two(c.lo), fma(x, ch, two(kGrid) - q));
    const float2 qs = split(q);
    const unsigned b0 = __float_as_uint(qs.x), b1 = __float_as_uint(qs.y);
    const float2 p0 = power(b0 % kPowers), p1 = power(b1 % kPowers);
    const Two u = r + two(p0.y, p1.y);
    const Two p = u * fma(u, fma(u, two(0.055504109f), two(0.24022651f)), two(0.69314718f));
    const Two h = two(__uint_as_float(__float_as_uint(p0.x) + ((b0 & ~(kPowers - 1u)) << 13)),
                      __uint_as_float(__float_as_uint(p1.x) + ((b1 & ~(kPowers - 1u)) << 13)));
    // (a: a whole number within 1 of h + h p; what h has over it is exact)
    const Two a = fma(h, p, h + kRound);
    const Two left = fma(h, p, h - (a - kRound));
    const float2 as = split(a), rs = split(fma(left, two(4194304.f), kRound));
    high[0] = __float_as_uint(as.x), high[1] = __float_as_uint(as.y);
    rest[0] = __float_as_uint(rs.x), rest[1] = __float_as_uint(rs.y);
  }
  // The entry of low bits i, from the table of make_powers.
  __device__ __forceinline__ float2 entry(int i, const float2* of) const {
    static_assert(kPowers == 1 << 10, "a shift by 23 - 10 takes the other bits to the exponent's place");
    const float x = m - base, q = fmaf(x, c.hi, kGrid), r = fmaf(x, c.lo, fmaf(x, c.hi, kGrid - q));
    const unsigned from = static_cast<unsigned>(i) - __float_as_uint(q), k = from % kPowers;
    return make_float2(__uint_as_float(__float_as_uint(of[k].x) + (22u << 23) + ((from - k) << 13)), -(r + of[k].y));
  }
  __device__ __forceinline__ static unsigned long long join(unsigned high, unsigned rest) {
    return static_cast<unsigned long long>(high - kBits) * 4194304ull + static_cast<long long>(static_cast<int>(rest - kBits));
  }
  __device__ __forceinline__ float low() const { return m - 46.f / c.hi * 1.0001f; }
};

// ceil(p S) for p in [0, 1), at least 1.
__device__ __forceinline__ unsigned long long share_of(float p, unsigned long long S) {
  const uint32_t b = __float_as_uint(p);
  const int e = static_cast<int>(b >> 23);
  const unsigned long long f = e ? (b & 0x7fffffu) | 0x800000u : b & 0x7fffffu;
  const int shift = 150 - (e ? e : 1);                   // p = f 2^-shift, shift >= 24
  const unsigned long long lo = S * f, hi = __umul64hi(S, f);
  unsigned long long t;
  if (shift < 64)
    t = (hi << (64 - shift)) + (lo >> shift) + ((lo & ((1ull << shift) - 1)) ? 1 : 0);
  else
    t = shift < 128 ? (hi >> (shift - 64)) + 1 : 1;      // (one too many where nothing is left over: below 2^-40 of S)
  return t ? t : 1;
}

// Tokens of the order up to one of them (all: those above -inf).
struct Upto {
  float x;
  int i;
  // (of a row that is lost; an index within a slice is above -kMaxVocab)
  static __device__ __forceinline__ Upto lost_row() { return {0.f, -0x7fffffff}; }
  __device__ __forceinline__ bool lost() const { return i == -0x7fffffff; }
  __device__ __forceinline__ bool has(float v, int at) const { return v > x || (v == x && at <= i); }
};

__device__ __forceinline__ unsigned long long warp_sum_u64(unsigned long long v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

}  // namespace
}  // namespace dvi
