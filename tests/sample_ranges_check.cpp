// Checks the ranges of logits that sample.hip gathers by against the order of the
// values: prints what is wrong, and nothing otherwise.
#include "sample_ranges.h"

#include <cstdio>
#include <cstdlib>
#include <vector>

using namespace dptq::sampling;

static int wrong = 0;
static void expect(bool ok, const char* what, Range r, uint32_t of) {
  if (!ok && ++wrong <= 20) std::printf("%s: range %08x to %08x, %08x\n", what, r.lo, r.hi, of);
}

// Of fp16 bits, none of them NaN's.
static float half_value(int h) {
  const int e = h >> 10 & 31, m = h & 0x3FF;
  float x = e == 31 ? __builtin_inff() : e ? (float)(0x400 + m) * __builtin_powif(2.0f, e - 25) : (float)m * 0x1p-24f;
  return h & 0x8000 ? -x : x;
}

// What a value is compared with: fp32 values as they are, fp16 ones clamped to
// the range's, where it has any, which leaves those in it as they are.
static bool marked(float v, Range r) { return v >= value_of(r.lo) && v <= value_of(r.hi); }
static bool marked_half(int h, HalfRange in) {
  const int v = h & 0x8000 ? -(h & 0x7FFF) : h;
  const int up = v > in.least ? v : in.least, c = up < in.most ? up : in.most;
  return in.least <= in.most && c == v;
}

// The stretches that a range's tokens, or two ranges', the second above the first,
// are sorted by: in their order, and within bounds for any key.
static void check_buckets(Range r, Range above, const std::vector<int>& halves) {
  const bool two = above.lo <= above.hi;
  const Buckets b = buckets_of(Range{r.lo, two ? above.hi : r.hi}, two ? above.lo : 0, two ? above.lo - r.hi - 1 : 0);
  const uint32_t last = two ? above.hi : r.hi;
  expect(bucket_of(b, last) == 0, "first stretch", r, bucket_of(b, last));
  uint32_t before = 0;
  for (int i = 0; i <= 64; ++i) {   // keys of both ranges, descending
    const Range& in = two && i <= 32 ? above : r;
    const uint32_t span = in.hi - in.lo, step = two ? i <= 32 ? i : i - 33 : i, steps = two ? i <= 32 ? 32 : 31 : 64;
    const uint32_t at = bucket_of(b, in.hi - (uint32_t)((uint64_t)span * step / steps));
    expect(at >= before && at < (uint32_t)kBins, "stretch", r, at);
    before = at;
  }
  for (int h : halves) expect(bucket_of(b, key_of(half_value(h))) < (uint32_t)kBins, "any key's stretch", r, h);
  for (uint32_t k : {0u, 1u, r.lo - 1, last + 1, 0x7FFFFFFFu, 0xFFFFFFFFu})
    expect(bucket_of(b, k) < (uint32_t)kBins, "any key's stretch", r, k);
}

static void check(Range r, const std::vector<int>& halves) {
  expect(r.lo <= r.hi && key_of(value_of(r.lo)) == r.lo && key_of(value_of(r.hi)) == r.hi, "ends", r, 0);
  // Values around both ends, and around zero.
  for (uint32_t end : {r.lo, r.hi, 0x7FFFFFFEu, 0x80000000u, 0x80000001u})
    for (int d = -2; d <= 2; ++d) {
      const uint32_t k = end + d;
      if (k < kLowestKey || k > 0xFF800000u) continue;
      const float v = value_of(k);   // -0 too
      expect(marked(v, r) == (key_of(v) >= r.lo && key_of(v) <= r.hi), "value", r, k);
    }
  const HalfRange in = halves_of(r);
  for (int h : halves) {
    const uint32_t k = key_of(half_value(h));
    expect(marked_half(h, in) == (k >= r.lo && k <= r.hi), "fp16 value", r, h);
  }
  check_buckets(r, Range{1, 0}, halves);
}

int main() {
  std::vector<int> halves;
  for (int h = 0; h < 0x10000; ++h)
    if ((h & 0x7FFF) <= 0x7C00 && h != 0xFC00) halves.push_back(h);   // not masked
  uint32_t next = kLowestKey;
  for (int bin = 0; bin < kBins; ++bin) {
    const Range r = range_of(bin);
    // No key of a value lies between two bins.
    expect(r.lo == next || (next == 0x7FFFFFFFu && r.lo == 0x80000000u), "gap", r, next);
    next = r.hi + 1;
    expect(bin_of(r.lo) == bin && bin_of(r.hi) == bin, "bin", r, bin);
    check(r, halves);
  }
  expect(next == 0xFF800001u, "last", range_of(kBins - 1), next);
  for (int h : halves) {
    const float v = half_value(h);
    const Range r = range_of(bin_of(v));
    expect(key_of(v) >= r.lo && key_of(v) <= r.hi, "bin of a value", r, h);
  }
  // Stretches of bins, as narrowing cuts them: at both ends and anywhere.
  std::srand(1);
  for (int i = 0; i < 1500; ++i) {
    Range r = range_of(i % 3 == 0 ? kBins / 2 - 1 : i % 3 == 1 ? kBins / 2 : std::rand() % kBins);
    do {
      int shift = 0;
      while ((r.hi - r.lo) >> shift >= (uint32_t)kBins) ++shift;
      const uint32_t last = (r.hi - r.lo) >> shift;
      const uint32_t j = std::rand() % 3 == 0 ? 0 : std::rand() % 2 ? last : (uint32_t)std::rand() % (last + 1);
      r.lo += j << shift;
      const uint32_t end = r.lo + ((1u << shift) - 1);
      r.hi = r.hi < end ? r.hi : end;
      check(r, halves);
    } while (r.lo < r.hi);
  }
  for (int i = 0; i < 300; ++i) {
    const int a = std::rand() % kBins, c = std::rand() % kBins, low = a < c ? a : c, high = a < c ? c : a;
    if (low == high) continue;
    const int top = std::rand() % (high - low) + low + 1;
    check_buckets(range_of(low), Range{range_of(top).lo, range_of(high).hi}, halves);
  }
  return wrong != 0;
}
