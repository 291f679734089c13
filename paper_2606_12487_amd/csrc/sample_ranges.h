// The order of logits and its parts, as sample.hip counts and gathers them:
// pure functions of 32-bit keys (no HIP, so that they can be checked without a
// GPU).
#pragma once

#include <stdint.h>

namespace dptq {
namespace sampling {

// Values as integers in their order; -0 is 0, so that no value has the key
// 0x7FFFFFFF.
constexpr uint32_t kLowestKey = 0x00800000u;   // of -FLT_MAX; what is not masked is this or above
constexpr uint32_t key_of(float x) {
  const uint32_t u = __builtin_bit_cast(uint32_t, x + 0.0f);
  return u ^ (u >> 31 ? 0xFFFFFFFFu : 0x80000000u);
}
constexpr float value_of(uint32_t k) {
  return __builtin_bit_cast(float, k ^ (k >> 31 ? 0x80000000u : 0xFFFFFFFFu));
}

// Bins: five bits of the mantissa and 16 octaves, 2^-6 to 2^10, for each sign;
// smaller magnitudes in the bins at zero, larger ones in the outermost.
constexpr int kBinBits = 10, kBins = 1 << kBinBits;
constexpr int kBinShift = 18, kBinBase = (127 - 6) << 5;
// Of a value that counts, and of its key.
constexpr int bin_of(float x) {
  const uint32_t u = __builtin_bit_cast(uint32_t, x + 0.0f);   // -0 is 0
  const int q = (int)(u << 1 >> (kBinShift + 1)) - kBinBase;
  const int least = q > 0 ? q : 0, c = least < kBins / 2 - 1 ? least : kBins / 2 - 1;
  return c ^ ((int)u >> 31 & (kBins - 1)) ^ kBins / 2;   // negative: kBins / 2 - 1 - c
}
constexpr int bin_of(uint32_t k) { return bin_of(value_of(k)); }

// Keys lo to hi.  Values are compared with those of lo and hi, so neither may be
// 0x7FFFFFFF: as a value that is -0, which 0 is equal to.
struct Range {
  uint32_t lo, hi;
};
constexpr Range range_of(int bin) {
  const bool positive = bin >= kBins / 2;
  const int c = positive ? bin - kBins / 2 : kBins / 2 - 1 - bin;
  const uint32_t a = c == 0 ? 0 : (uint32_t)(c + kBinBase) << kBinShift;
  const uint32_t b = c == kBins / 2 - 1 ? 0x7F800000u : ((uint32_t)(c + kBinBase + 1) << kBinShift) - 1;
  if (positive) return Range{a | 0x80000000u, b | 0x80000000u};
  // Magnitudes a to b, negative; from the smallest one on, not from 0.
  return Range{b == 0x7F800000u ? kLowestKey : 0x7FFFFFFFu - b, 0x7FFFFFFFu - (a ? a : 1)};
}

// The largest magnitude of an fp16 number, as its bits, that is not above that of
// the fp32 number with bits a (none of the sign), and the smallest not below.
constexpr int half_within(uint32_t a) {
  if (a >= 0x7F800000u) return 0x7C00;                   // infinity
  if (a >= 0x477FE000u) return 0x7BFF;                   // 65504
  if (a >= 0x38800000u) return (int)((a - 0x38000000u) >> 13);
  if (a < 0x33800000u) return 0;                         // below 2^-24
  return (int)((0x800000u | (a & 0x7FFFFFu)) >> (126 - (a >> 23)));
}
constexpr int half_beyond(uint32_t a) { return a ? half_within(a - 1) + 1 : 0; }

// The fp16 numbers of a range: least to most, as magnitudes with their sign; least
// above most where none lies in it.
struct HalfRange {
  int least, most;
};
constexpr HalfRange halves_of(Range r) {
  const uint32_t lo = r.lo >> 31 ? r.lo & 0x7FFFFFFFu : 0x7FFFFFFFu - r.lo;
  const uint32_t hi = r.hi >> 31 ? r.hi & 0x7FFFFFFFu : 0x7FFFFFFFu - r.hi;
  return HalfRange{r.lo >> 31 ? half_beyond(lo) : -half_within(lo), r.hi >> 31 ? half_within(hi) : -half_beyond(hi)};
}
constexpr uint16_t half_bits(int magnitude) {
  return (uint16_t)(magnitude < 0 ? 0x8000 - magnitude : magnitude);
}

// Which of kBins stretches of a range (without the `gap` keys below `split`), from
// its upper end, a key is in.  A key that is not in the range, as of a row that
// changes between two readings, gets one of them too.
struct Buckets {
  Range r;
  uint32_t split, gap;
  int shift;
};
constexpr Buckets buckets_of(Range r, uint32_t split, uint32_t gap) {
  const uint32_t keys = r.hi - r.lo - gap;   // and one
  const int bits = keys ? 32 - __builtin_clz(keys) : 0;
  return Buckets{r, split, gap, bits > kBinBits ? bits - kBinBits : 0};
}
constexpr uint32_t bucket_of(const Buckets& b, uint32_t key) {
  const uint32_t i = (b.r.hi - key - (key < b.split ? b.gap : 0)) >> b.shift;
  return i < kBins ? i : kBins - 1;
}

}  // namespace sampling
}  // namespace dptq
