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
// table of 128, and 2^-g = 1 + z + z^2 / 2 + z^3 / 6, z = -g ln 2, up to 2^-38.
// The float operations round z and its series to about 2^-32.5, the table and the
// product are rounded to units of 2^-30 of a number in (1/2, 1].  So a weight is
// off by some 2^-30 of itself, and by less than one unit from being cut to them.
struct SampleScale {
  float hi, lo;  // log2(e) / T
  int shift;
};
constexpr int kSampleTable = 128;
constexpr float kSampleDead = 40.f;  // weights below 2^-40 are zero
constexpr float kSampleMagic = 12582912.f;  // 1.5 * 2^23: adding it rounds to a whole number

// Units of a row of `vocab` logits: their sum stays below 2^63.
inline int sample_shift(long long vocab) {
  int bits = 0;
  while ((1ll << bits) < vocab) ++bits;
  return 62 - bits < 44 ? 62 - bits : 44;
}
EBD_HD SampleScale sample_scale(float temperature, int shift) {
  // 1 / T within float's range whatever T is
  const double t = temperature < 1e-30f ? 1e-30 : temperature > 1e30f ? 1e30 : static_cast<double>(temperature);
  const double c = 1.4426950408889634 / t;
  const float hi = static_cast<float>(c);
  return {hi, static_cast<float>(c - hi), shift};
}
struct SampleEntry {
  uint32_t fixed;  // 2^(-j / 128) in units of 2^-30
  float scaled;    // the same, a float
};
EBD_HD SampleEntry sample_entry(int j) {
  const double x = exp2(-j / 128.0) * 1073741824.0;
  return {static_cast<uint32_t>(x + 0.5), static_cast<float>(x)};
}
// y, rounded: it grows as l falls, and decides alone which weights are zero
EBD_HD float sample_depth(float m, float l, const SampleScale& c) { return (m - l) * c.hi; }

EBD_HD uint64_t sample_weight(float m, float l, const SampleScale& c, const SampleEntry* table) {
  const float s = m - l;
  const float p = s * c.hi;
  if (!(p <= kSampleDead)) return 0;
  const float b = s - m;
  const float d = (m - (s - b)) - (l + b);  // s + d = m - l exactly
  const float e = fmaf(s, c.hi, -p) + fmaf(s, c.lo, d * c.hi);
  const float t = fmaf(p, 128.f, kSampleMagic);
  const int k = static_cast<int>(f32_bits(t) & 0x3FFFFFu);
  const float g = fmaf(t - kSampleMagic, -0.0078125f, p) + e;
  const float z = g * -0.693147181f;
  const float x = z * fmaf(z, fmaf(z, 0.166666667f, 0.5f), 1.f);
  const SampleEntry q = table[k & (kSampleTable - 1)];
  const uint32_t w = q.fixed + (f32_bits(fmaf(q.scaled, x, kSampleMagic)) - f32_bits(kSampleMagic));
  return (static_cast<uint64_t>(w) << 32) >> (62 - c.shift + (k >> 7));
}

// Least sum that a kept share p of `total` asks for: at least one unit.
EBD_HD uint64_t sample_share(float p, uint64_t total) {
  if (!(p > 0.f)) return 1;
  const double x = ceil(static_cast<double>(p) * static_cast<double>(total));
  const uint64_t t = static_cast<uint64_t>(x);
  return t < 1 ? 1 : t > total ? total : t;
}
// The unit that u in [0, 1) points at: token = the first whose sum passes it.
EBD_HD uint64_t sample_point(float u, uint64_t total) {
  const uint64_t t = static_cast<uint64_t>(static_cast<double>(u) * static_cast<double>(total));
  return t < total ? t : total - 1;
}
// Least logit with weight >= q of the largest's (q > 0).
EBD_HD float sample_floor(float m, float temperature, float q) {
  if (q >= 1.f) return m;
  const double x = static_cast<double>(m) + static_cast<double>(temperature) * log(static_cast<double>(q));
  float f = static_cast<float>(x);
  if (static_cast<double>(f) < x) f = nextafterf(f, INFINITY);
  return f < m ? f : m;
}

}  // namespace ebd
