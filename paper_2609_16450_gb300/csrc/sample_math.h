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

// Whole numbers in the order of the floats they stand for (no NaN, no -0).
EBD_HD uint32_t order_key(float x) {
  const uint32_t b = f32_bits(x);
  return b ^ ((b >> 31) != 0 ? 0xFFFFFFFFu : 0x80000000u);
}
EBD_HD float order_value(uint32_t k) { return f32_of((k >> 31) != 0 ? k ^ 0x80000000u : ~k); }

// The weight of logit l is w = exp((l - m) / T) in whole units of 2^-shift, m the
// row's largest logit, and 0 below 2^-40.  Sums of such weights are exact in any
// order, so that a token's border in them is one number wherever it is computed.
//
// w = 2^-y with y = (m - l) log2(e) / T as the sum of two floats, p + e: m - l is
// exact in two floats, and so is its product with the rounded factor.  Then y = k /
// 128 + g with |g| <= 2^-8 (and e): 2^(-k / 128) is 2^(-(k >> 7)) times an entry of a
// table of 128, and 2^-g = 1 + x, x a cubic in g that leaves out 2^-38.  The float
// operations round g and the cubic by about 2^-32.5, the table and the product are
// rounded to units of 2^-30 of a number in (1/2, 1].  So a weight is off by some
// 2^-30 of itself, and by less than one unit from being cut to them.
struct SampleScale {
  float hi, lo;  // log2(e) / T
  int shift;
};
constexpr int kSampleTable = 128;
constexpr float kSampleDead = 40.f;  // weights below 2^-40 are zero
constexpr float kSampleMagic = 12582912.f;  // 1.5 * 2^23: adding it rounds to a whole number
constexpr uint32_t kSampleMagicBits = 0x4B400000u;
// 2^-g - 1 = g (c1 + g (c2 + g c3)): -ln 2, (ln 2)^2 / 2, -(ln 2)^3 / 6
constexpr float kSampleC1 = -0.693147181f, kSampleC2 = 0.240226507f, kSampleC3 = -0.0555041087f;

// Units of a row of `vocab` logits: their sum stays below 2^63.
inline int sample_shift(long long vocab) {
  int bits = 0;
  while ((1ll << bits) < vocab) ++bits;
  return 62 - bits < 44 ? 62 - bits : 44;
}
// 1 / T stays within float's range
EBD_HD float sample_temperature(float t) { return t < 1e-30f ? 1e-30f : t > 1e30f ? 1e30f : t; }
EBD_HD SampleScale sample_scale(float temperature, int shift) {
  const double c = 1.4426950408889634 / static_cast<double>(temperature);
  const float hi = static_cast<float>(c);
  return {hi, static_cast<float>(c - hi), shift};
}
// 2^(-j / 128) in units of 2^-30
EBD_HD uint32_t sample_entry(int j) { return static_cast<uint32_t>(exp2(-j / 128.0) * 1073741824.0 + 0.5); }
// the same entry as a float: its leading bits
EBD_HD float sample_entry_float(uint32_t q) { return f32_of((155u << 23) + (q >> 6)); }
// y, rounded: it grows as l falls, and decides alone which weights are zero
EBD_HD float sample_depth(float m, float l, const SampleScale& c) { return (m - l) * c.hi; }

// The weight before it is cut, w 2^(-30 - k), w in (2^29, 2^30]; k = 64 for none.
struct SampleTerm {
  uint32_t w;
  int k;
};
EBD_HD SampleTerm sample_term(float m, float l, const SampleScale& c, const uint32_t* table) {
  const float s = m - l;
  const float p = s * c.hi;
  if (!(p <= kSampleDead)) return {0, 64};
  const float b = s - m;
  const float d = (m - (s - b)) - (l + b);  // s + d = m - l exactly
  const float e = fmaf(d, c.hi, fmaf(s, c.lo, fmaf(s, c.hi, -p)));
  const float t = fmaf(p, 128.f, kSampleMagic);
  const uint32_t k = f32_bits(t) - kSampleMagicBits;
  const float g = fmaf(t - kSampleMagic, -0.0078125f, p) + e;
  const float x = g * fmaf(g, fmaf(g, kSampleC3, kSampleC2), kSampleC1);
  const uint32_t q = table[k & (kSampleTable - 1)];
  const uint32_t w = q + (f32_bits(fmaf(sample_entry_float(q), x, kSampleMagic)) - kSampleMagicBits);
  return {w, static_cast<int>(k >> 7)};
}
EBD_HD uint64_t sample_weight(float m, float l, const SampleScale& c, const uint32_t* table) {
  const SampleTerm t = sample_term(m, l, c, table);
  return t.w != 0 ? (static_cast<uint64_t>(t.w) << 32) >> (62 - c.shift + t.k) : 0;
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
// Least logit with weight >= q of the largest's, for (hi, lo) = T ln q in two floats.
EBD_HD float sample_floor(float m, float hi, float lo) {
  const float s = m + hi, b = s - m;
  const float r = ((m - (s - b)) + (hi - b)) + lo;  // s + r = m + T ln q
  const float f = s + r;
  return r - (f - s) > 0.f ? order_value(order_key(f + 0.f) + 1) : f;
}

}  // namespace ebd
