// Arithmetic of the sampler (k_sample.cu), for the kernel and, compiled by a host
// compiler, for tests: a token's weight, the order of logits, the kept share's
// border.
#pragma once
#include <cmath>
#include <cstdint>
#include <cstring>

#ifdef __CUDACC__
#define EBD_HD __host__ __device__ __forceinline__
#else
#define EBD_HD inline
#endif

namespace ebd {

EBD_HD uint32_t f32_bits(float x) {
#ifdef __CUDA_ARCH__
  return __float_as_uint(x);
#else
  uint32_t b;
  std::memcpy(&b, &x, 4);
  return b;
#endif
}
EBD_HD float f32_of(uint32_t b) {
#ifdef __CUDA_ARCH__
  return __uint_as_float(b);
#else
  float x;
  std::memcpy(&x, &b, 4);
  return x;
#endif
}

// A product rounded by itself: never part of a fused multiply-add, whatever a compiler is
// allowed.
EBD_HD float rounded_product(float a, float b) {
#ifdef __CUDA_ARCH__
  return __fmul_rn(a, b);
#else
  const volatile float p = a * b;
  return p;
#endif
}

// Whole numbers in the order of the floats they stand for (no NaN, no -0).
EBD_HD uint32_t order_key(float x) {
  const uint32_t b = f32_bits(x);
  return b ^ ((b >> 31) != 0 ? 0xFFFFFFFFu : 0x80000000u);
}
EBD_HD float order_value(uint32_t k) { return f32_of((k >> 31) != 0 ? k ^ 0x80000000u : ~k); }

// The weight of logit l is w = exp((l - m) / T) in whole units of 2^-43, m the row's
// largest logit, and 0 below 2^-40.  Sums of such weights are exact in any order, so
// that a token's border in them is one number wherever it is computed.
//
// w = 2^(-y / 128) with y = (m - l) 128 log2(e) / T as the sum of two floats, p + e: m -
// l is exact in two floats, and so is its product with the rounded factor.  Then y = k +
// z with |z| <= 1/2 (and e): 2^(-k / 128) is 2^(-(k >> 7)) times an entry of a table of
// 128, a float v and what it is off by, relative to it; 2^(-z / 128) - 1 is a cubic in z
// that leaves out 2^-38, and starts from that.  w = v + v x is rounded to units of
// 2^-21, h (v first, then v + v x, so that 2^-21 may be left), and what is left to
// units of 2^-43, all in float operations that are exact but for those roundings:
// whole-number shifts and additions have half their rate.
// The roundings of z and x make a weight off by some 2^-31 of itself, and the last two
// by 5/8 of a unit.
struct SampleScale {
  float hi, lo;  // 128 log2(e) / T
};
constexpr int kSampleVocab = 1 << 20;  // sums of fewer weights fit 64 bits
constexpr int kSampleTable = 128;
constexpr float kSampleDead = 40.f * kSampleTable;  // weights below 2^-40 are zero
constexpr float kSampleMagic = 12582912.f;  // 1.5 * 2^23: adding it rounds to a whole number,
constexpr float kSampleHigh = 6.f;          // 1.5 * 2^2: to a unit of 2^-21,
constexpr float kSampleLow = 1.430511474609375e-6f;  // 1.5 * 2^-20: to one of 2^-43
constexpr float kSampleUnits = 8796093022208.f;      // 2^43
// 2^(-z / 128) - 1 = z (c1 + z (c2 + z c3)): -ln 2, (ln 2)^2 / 2, -(ln 2)^3 / 6 with a
// factor of 2^-7 for every z
constexpr float kSampleC1 = -0.693147181f / 128, kSampleC2 = 0.240226507f / 16384, kSampleC3 = -0.0555041087f / 2097152;

// 1 / T stays within float's range
EBD_HD float sample_temperature(float t) { return t < 1e-30f ? 1e-30f : t > 1e30f ? 1e30f : t; }
EBD_HD SampleScale sample_scale(float temperature) {
  const double c = 1.4426950408889634 * kSampleTable / static_cast<double>(temperature);
  const float hi = static_cast<float>(c);
  return {hi, static_cast<float>(c - hi)};
}
struct SampleEntry {
  uint32_t bits;  // of v = 2^(-j / 128), plus j << 16: less k << 16 they are those of v 2^(-(k >> 7))
  float off;      // (2^(-j / 128) - v) / v
};
inline SampleEntry sample_entry(int j) {
  const double x = std::exp2(-j / 128.0);
  const float v = static_cast<float>(x);
  return {f32_bits(v) + (static_cast<uint32_t>(j) << 16), static_cast<float>((x - v) / v)};
}
// y, rounded: it grows as l falls, and decides alone which weights are zero
EBD_HD float sample_depth(float m, float l, const SampleScale& c) { return rounded_product(m - l, c.hi); }

// w = v + v x of a logit that has weight
struct SampleTerm {
  float v, x;
};
EBD_HD SampleTerm sample_term(float m, float l, const SampleScale& c, const SampleEntry* table) {
  const float s = m - l;
  const float b = s - m;
  const float d = (m - (s - b)) - (l + b);  // s + d = m - l exactly
  const float p = rounded_product(s, c.hi);  // e holds what this rounding leaves out
  const float e = fmaf(d, -c.hi, fmaf(s, -c.lo, fmaf(s, -c.hi, p)));  // -e above
  const float t = p + kSampleMagic;
  const float z = (p - (t - kSampleMagic)) - e;
  const SampleEntry q = table[f32_bits(t) & (kSampleTable - 1)];
  return {f32_of(q.bits - (f32_bits(t) << 16)), fmaf(z, fmaf(z, fmaf(z, kSampleC3, kSampleC2), kSampleC1), q.off)};
}
// the same in whole numbers of 2^-21 and of 2^-43
struct SampleParts {
  float high, low;
};
EBD_HD SampleParts sample_parts(const SampleTerm& w) {
  const float h = fmaf(w.v, w.x, w.v + kSampleHigh) - kSampleHigh;
  return {h, (fmaf(w.v, w.x, w.v - h) + kSampleLow) - kSampleLow};
}
EBD_HD uint64_t sample_weight(float m, float l, const SampleScale& c, const SampleEntry* table) {
  if (!(sample_depth(m, l, c) <= kSampleDead)) return 0;
  const SampleParts w = sample_parts(sample_term(m, l, c, table));
  return static_cast<uint64_t>(static_cast<int64_t>(w.high * 2097152.f) * 4194304 + static_cast<int64_t>(w.low * kSampleUnits));
}

// total * x for a float x in [0, 1), cut or rounded up to a whole number: exactly.
EBD_HD uint64_t sample_part(float x, uint64_t total, bool up) {
  const uint32_t b = f32_bits(x), e = b >> 23;
  const uint64_t mant = e != 0 ? (b & 0x7FFFFFu) | 0x800000u : b;  // x = mant * 2^-k
  const int k = 150 - static_cast<int>(e != 0 ? e : 1);              // 24 .. 149
#ifdef __CUDA_ARCH__
  const uint64_t hi = __umul64hi(total, mant);
#else
  const uint64_t hi = static_cast<uint64_t>((static_cast<unsigned __int128>(total) * mant) >> 64);
#endif
  const uint64_t lo = total * mant;
  uint64_t whole, rest;
  if (k < 64) {
    whole = lo >> k | hi << (64 - k);
    rest = lo << (64 - k);
  } else {  // hi is below 2^24
    whole = k < 88 ? hi >> (k - 64) : 0;
    rest = lo | (hi - (k < 88 ? whole << (k - 64) : 0));
  }
  return whole + (up && rest != 0 ? 1 : 0);
}
// Least sum that a kept share p < 1 of `total` asks for: at least one unit.
EBD_HD uint64_t sample_share(float p, uint64_t total) {
  const uint64_t t = p > 0.f ? sample_part(p, total, true) : 0;
  return t < 1 ? 1 : t;
}
// The unit that u in [0, 1) points at: token = the first whose sum passes it.
EBD_HD uint64_t sample_point(float u, uint64_t total) { return sample_part(u, total, false); }
// Least logit with weight >= q of the largest's, for (hi, lo) = T ln q in two floats;
// the lowest float where that lies below float's range (m + hi = -inf would make the rest
// NaN: what is left of it then is in r).
EBD_HD float sample_floor(float m, float hi, float lo) {
  const float s = fmaxf(m + hi, -3.402823466e38f), b = s - m;
  const float r = ((m - (s - b)) + (hi - b)) + lo;  // s + r = m + T ln q
  const float f = s + r;
  return r - (f - s) > 0.f ? order_value(order_key(f + 0.f) + 1) : f;
}

}  // namespace ebd
