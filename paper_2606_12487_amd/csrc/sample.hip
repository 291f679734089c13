// One token of each row of logits x [M, V] under temperature, top-k, top-p and
// min-p, from a given uniform number u a row.
//
// The tokens of a row in order: larger logits first, equal ones by index.  With
// w = exp((x - max x) / T), sums of w in that order:
//
//   K1 = the first top_k tokens,  W1 = their sum
//   K2 = those of K1 before which the sum is below top_p * W1 (the first always)
//   K3 = those of K2 with w >= min_p (the first always),  W3 = their sum
//   token = the first one up to which the sum is above u * W3;  prob = w / W3
//
// Every step is a border in the order, "the first n tokens", given by a count,
// by a sum or by a value; so no step needs the row sorted, only the place of a
// border.  A histogram of the row (counts, and sums of w as integers of 2^-46,
// which no order of additions changes) over 1024 bins of the value, a
// 1/32 of an octave wide, says which bin a border is in; that bin's tokens, a few
// hundred as a rule, are gathered and sorted, and their running sum gives the
// place.  A bin of more than 2048 tokens is cut into 1024 again and again until
// it is small or all its values are equal, when index and sum are arithmetic.
// Where everything down to the lowest border is at most 2048 tokens, which
// top-k and top-p mostly leave, they are gathered once for all borders.
//
// w in 64 bits: with 131072 tokens of like weight a relative error of 2^-24 in
// the sums would change one token in a hundred.  2^t = 2^n (1 + f q(f)) with n
// the nearest integer and q the interpolant of degree 8 at Chebyshev's nodes on
// [-1/2, 1/2], to 4e-14.
#include "internal.h"

namespace dptq {
namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kBins = 1024;       // one a thread
constexpr int kCap = 2048;        // tokens that are sorted at once
constexpr int kMinPart = 8192;    // logits of a part of a row, at least

// Values as integers in their order; -0 is 0.
constexpr uint32_t kLowestKey = 0x00800000u, kHighestKey = 0xFF800000u;   // -FLT_MAX to +inf: what counts
__device__ __forceinline__ uint32_t key_of(float x) {
  const uint32_t u = __float_as_uint(x + 0.0f);
  return u ^ (u >> 31 ? 0xFFFFFFFFu : 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t k) {
  return __uint_as_float(k ^ (k >> 31 ? 0x80000000u : 0xFFFFFFFFu));
}
__device__ __forceinline__ bool counts(uint32_t k) { return k - kLowestKey <= kHighestKey - kLowestKey; }

// Bins: five bits of the mantissa and 16 octaves, 2^-6 to 2^10, for each sign;
// smaller magnitudes in the bins at zero, larger ones in the outermost.
constexpr int kBinShift = 18, kBinBase = (127 - 6) << 5;
__device__ __forceinline__ int bin_of(uint32_t k) {
  const bool positive = k >> 31;
  const int q = (int)(((positive ? k : ~k) & 0x7FFFFFFFu) >> kBinShift) - kBinBase;
  const int c = min(max(q, 0), kBins / 2 - 1);
  return positive ? kBins / 2 + c : kBins / 2 - 1 - c;
}
struct Range {
  uint32_t lo, hi;   // keys, both in it
};
__device__ __forceinline__ Range range_of(int bin) {
  const bool positive = bin >= kBins / 2;
  const int c = positive ? bin - kBins / 2 : kBins / 2 - 1 - bin;
  const uint32_t a = c == 0 ? 0 : (uint32_t)(c + kBinBase) << kBinShift;
  const uint32_t b = c == kBins / 2 - 1 ? 0x7F800000u : ((uint32_t)(c + kBinBase + 1) << kBinShift) - 1;
  if (positive) return Range{a | 0x80000000u, b | 0x80000000u};
  return Range{b == 0x7F800000u ? kLowestKey : 0x7FFFFFFFu - b, 0x7FFFFFFFu - a};   // magnitudes a to b, negative
}

// 2^((x - m) c) in 64 bits, for x <= m.
__device__ __forceinline__ double weight(float x, float m, double c) {
  const double t = fmax(((double)x - (double)m) * c, -2000.0);
  const double n = __builtin_rint(t), f = t - n;
  double q = __builtin_fma(f, 0x1.b639ab2e49ae8p-24, 0x1.63d1341b008a0p-20);
  q = __builtin_fma(f, q, 0x1.ffcb942c7e385p-17);
  q = __builtin_fma(f, q, 0x1.4308ac87f8c3cp-13);
  q = __builtin_fma(f, q, 0x1.5d87fe872c528p-10);
  q = __builtin_fma(f, q, 0x1.3b2ab71819e07p-7);
  q = __builtin_fma(f, q, 0x1.c6b08d7047e27p-5);
  q = __builtin_fma(f, q, 0x1.ebfbdff823cfep-3);
  q = __builtin_fma(f, q, 0x1.62e42fefa39edp-1);
  q = __builtin_fma(f, q, 1.0);
  return __builtin_ldexp(q, (int)n);
}

// A weight in units of 2^-e, to the nearest: the sum with 2^52 leaves it in the
// mantissa.  unit = 2^e, e <= 46.
using u64 = unsigned long long;
__device__ __forceinline__ u64 fixed(double w, double unit) {
  return (u64)__double_as_longlong(__builtin_fma(w, unit, 0x1p52)) & 0xFFFFFFFFFFFFFull;
}

// Calls f(x[i], i) for lo <= i < hi over a workgroup; 16-byte loads where they
// are whole, U in flight.
template <int U, typename T, typename F>
__device__ __forceinline__ void for_logits(const T* x, int lo, int hi, const F& f) {
  constexpr int E = 16 / sizeof(T);
  const int start = lo - (int)((reinterpret_cast<uintptr_t>(x + lo) & 15) / sizeof(T));
  for (int64_t at = start; at < hi; at += (int64_t)U * kThreads * E) {
    uint4 v[U];
    int64_t i[U];
    bool whole[U];
#pragma unroll
    for (int n = 0; n < U; ++n) {
      i[n] = at + ((int64_t)n * kThreads + threadIdx.x) * E;
      whole[n] = i[n] >= lo && i[n] + E <= hi;
      if (whole[n]) v[n] = *reinterpret_cast<const uint4*>(x + i[n]);
    }
#pragma unroll
    for (int n = 0; n < U; ++n) {
      if (whole[n]) {
        const T* const e = reinterpret_cast<const T*>(&v[n]);
#pragma unroll
        for (int j = 0; j < E; ++j) f((float)e[j], (int)i[n] + j);
      } else {
        for (int j = 0; j < E; ++j)
          if (i[n] + j >= lo && i[n] + j < hi) f((float)x[i[n] + j], (int)(i[n] + j));
      }
    }
  }
}

struct SampleArgs {
  const void* x;
  int64_t ld, M;
  int V, splits, part;      // part: logits of a split
  double unit;              // 2^e of the sums of a row
  const float* u;
  const float *temperature, *top_p, *min_p;   // of each row, or nullptr and the value
  const int32_t* top_k;
  float temperature_all, top_p_all, min_p_all;
  int top_k_all;
  int64_t* tokens;
  float* probs;
  u64* mass;                // [M][splits][kBins]
  uint32_t* count;
  float* most;              // [M][splits]
};

// log2(e) / T; a greedy row (T = 0) is that of T = 1.
__device__ __forceinline__ double factor(const SampleArgs& a, int64_t row, bool* greedy) {
  const float t = a.temperature ? a.temperature[row] : a.temperature_all;
  *greedy = !(t > 0.0f);
  return 1.4426950408889634 / (*greedy ? 1.0 : (double)t);
}

struct Histogram {
  u64 mass[kBins];
  uint32_t count[kBins];
};

struct Shared {
  Histogram h;                 // of the row, then of a bin that is cut again
  double mass[kBins + 1];      // before bin kBins - 1 - j
  uint32_t count[kBins + 1];
  u64 list[kCap];              // key and ~index, in the order
  double sum[kCap];            // up to each
  double wave_d[kWaves];
  uint32_t wave_u[kWaves];
  float wave_f[kWaves];
  int n, found;
};

__device__ __forceinline__ void clear(Histogram& h) {
  h.mass[threadIdx.x] = 0;
  h.count[threadIdx.x] = 0;
}

__device__ __forceinline__ float block_max(float x, float* part) {
  for (int s = 32; s > 0; s >>= 1) x = fmaxf(x, __shfl_xor(x, s));
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = x;
  __syncthreads();
  x = part[threadIdx.x & (kWaves - 1)];
  for (int s = kWaves / 2; s > 0; s >>= 1) x = fmaxf(x, __shfl_xor(x, s));
  return x;
}

// The largest logit of [lo, hi), and their histogram relative to it.
template <typename T>
__device__ __forceinline__ float histogram(const T* x, int lo, int hi, double c, double unit, Histogram& h,
                                           float* part) {
  float m = -INFINITY;
  for_logits<4>(x, lo, hi, [&](float v, int) { m = fmaxf(m, v); });
  clear(h);
  m = block_max(m, part);   // its barrier is the histogram's too
  for_logits<1>(x, lo, hi, [&](float v, int) {
    const uint32_t k = key_of(v);
    if (!counts(k)) return;
    const int b = bin_of(k);
    atomicAdd(&h.count[b], 1u);
    atomicAdd(&h.mass[b], fixed(weight(v, m, c), unit));
  });
  __syncthreads();
  return m;
}

// Inclusive sums over the workgroup, in the order of the threads.
template <typename V>
__device__ __forceinline__ V block_scan(V x, V* part) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int s = 1; s < 64; s <<= 1) {
    const V y = __shfl_up(x, s);
    if (lane >= s) x += y;
  }
  if (lane == 63) part[wave] = x;
  __syncthreads();
  V before = 0;
  for (int w = 0; w < kWaves; ++w)
    if (w < wave) before += part[w];
  __syncthreads();
  return before + x;
}

// What a border is given by.
enum class By { kCount, kSumBelow, kKey, kSumAbove };
struct Border {
  By by;
  uint32_t n;      // kCount: the n-th token is the last before the border (n >= 1)
  double sum;      // kSumBelow: tokens before which the sum is below it;
                   // kSumAbove: the token up to which the sum is above it is the last
  uint32_t key;    // kKey: tokens of this key and above
};
// Where it is: tokens before it, their sum, and the last of them.
struct Place {
  uint32_t n;
  double sum;
  uint32_t key;
  int index;
};

template <typename T>
struct Selector {
  const T* x;
  int V;
  float m;
  double c, unit;
  Shared& s;
  // What the list holds: all tokens of a range, those before it.
  Range range;
  uint32_t before_n, held;
  double before_sum;

  __device__ __forceinline__ double weight_of(uint32_t key) const { return weight(value_of(key), m, c); }

  // The cumulative counts and sums of s.h, descending, after `n` tokens of sum `sum`.
  __device__ __forceinline__ void cumulate(uint32_t count, double mass, uint32_t n, double sum) {
    const uint32_t cn = block_scan(count, s.wave_u);
    const double cm = block_scan(mass, s.wave_d);
    s.count[threadIdx.x + 1] = n + cn;
    s.mass[threadIdx.x + 1] = sum + cm;
    if (threadIdx.x == 0) s.count[0] = n, s.mass[0] = sum;
    __syncthreads();
  }

  // Which of the cumulated bins (0: the first in the order) a border is in; the
  // last that is not empty where rounding leaves none.  kKey does not come here.
  __device__ __forceinline__ int bin_with(const Border& b) {
    const int j = threadIdx.x;
    if (j == 0) s.found = -1;
    __syncthreads();
    const uint32_t n0 = s.count[j], n1 = s.count[j + 1];
    const double m0 = s.mass[j], m1 = s.mass[j + 1];
    const bool here = b.by == By::kCount ? n0 < b.n && b.n <= n1
                    : b.by == By::kSumBelow ? m0 < b.sum && b.sum <= m1
                                            : m0 <= b.sum && b.sum < m1;
    if (here && n1 > n0) s.found = j;
    __syncthreads();
    int found = s.found;
    if (found < 0) {
      __syncthreads();
      if (n1 > n0) atomicMax(&s.found, j);
      __syncthreads();
      found = max(s.found, 0);
    }
    __syncthreads();
    return found;
  }

  // Gathers the tokens of a range, at most kCap, in their order, with their sums.
  __device__ __forceinline__ void load(Range r, uint32_t n, double sum) {
    if (threadIdx.x == 0) s.n = 0;
    __syncthreads();
    for_logits<4>(x, 0, V, [&](float v, int i) {
      const uint32_t k = key_of(v);
      if (k - r.lo > r.hi - r.lo) return;
      const int at = atomicAdd(&s.n, 1);
      if (at < kCap) s.list[at] = (u64)k << 32 | (uint32_t)~i;
    });
    __syncthreads();
    const int count = min(s.n, kCap);
    int size = 64;
    while (size < count) size *= 2;
    for (int i = count + threadIdx.x; i < size; i += kThreads) s.list[i] = 0;   // behind all
    __syncthreads();
    for (int k = 2; k <= size; k *= 2)
      for (int j = k / 2; j > 0; j /= 2) {
        const int i = threadIdx.x, a = 2 * i - (i & (j - 1)), b = a + j;
        if (i < size / 2) {
          const u64 p = s.list[a], q = s.list[b];
          if ((p < q) == ((a & k) == 0)) s.list[a] = q, s.list[b] = p;
        }
        __syncthreads();
      }
    const int a = 2 * threadIdx.x;
    const double w0 = a < count ? weight_of((uint32_t)(s.list[a] >> 32)) : 0.0;
    const double w1 = a + 1 < count ? weight_of((uint32_t)(s.list[a + 1] >> 32)) : 0.0;
    const double up_to = block_scan(w0 + w1, s.wave_d);
    s.sum[a] = sum + (up_to - w1);
    s.sum[a + 1] = sum + up_to;
    __syncthreads();
    range = r;
    before_n = n;
    before_sum = sum;
    held = (uint32_t)count;
  }

  // A border among the list's tokens.
  __device__ __forceinline__ Place in_list(const Border& b) {
    const int i = 2 * threadIdx.x;
    uint32_t n = 0;   // tokens of the list before the border
    if (b.by == By::kCount) {
      n = b.n - before_n;
    } else {
      int yes = 0;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int at = i + e;
        if (at >= (int)held) continue;
        if (b.by == By::kKey) yes += (uint32_t)(s.list[at] >> 32) >= b.key;
        else if (b.by == By::kSumAbove) yes += s.sum[at] <= b.sum;
        else yes += (at ? s.sum[at - 1] : before_sum) < b.sum;
      }
      const uint32_t all = block_scan((uint32_t)yes, s.wave_u);
      if (threadIdx.x == kThreads - 1) s.n = (int)all;
      __syncthreads();
      n = (uint32_t)s.n + (b.by == By::kSumAbove);
      __syncthreads();
    }
    n = min(n, held);
    Place p{before_n + n, n ? s.sum[n - 1] : before_sum, 0, -1};
    if (n) {
      p.key = (uint32_t)(s.list[n - 1] >> 32);
      p.index = (int)~(uint32_t)s.list[n - 1];
    }
    return p;
  }

  // A border among `count` equal values.
  __device__ __forceinline__ Place in_ties(const Border& b, uint32_t key, uint32_t n0, double sum0, uint32_t count) {
    const double w = weight_of(key);
    double n = count;
    if (b.by == By::kCount) n = (double)(b.n - n0);
    else if (b.by == By::kKey) n = key >= b.key ? n : 0.0;
    else if (b.by == By::kSumBelow) n = ceil((b.sum - sum0) / w);
    else n = floor((b.sum - sum0) / w) + 1.0;
    const uint32_t k = (uint32_t)fmax(fmin(n, (double)count), b.by == By::kSumAbove ? 1.0 : 0.0);
    Place p{n0 + k, sum0 + k * w, key, -1};
    if (k == 0) return p;
    // The k-th of them by index: each thread counts those of a stretch.
    const int stretch = (V + kThreads - 1) / kThreads;
    const int lo = min((int64_t)threadIdx.x * stretch, (int64_t)V), hi = min(lo + stretch, V);
    uint32_t mine = 0;
    for (int i = lo; i < hi; ++i) mine += key_of((float)x[i]) == key;
    const uint32_t up_to = block_scan(mine, s.wave_u);
    if (threadIdx.x == 0) s.found = -1;
    __syncthreads();
    if (up_to >= k && up_to - mine < k) {
      uint32_t at = up_to - mine;
      for (int i = lo; i < hi; ++i) {
        if (key_of((float)x[i]) != key) continue;
        if (++at == k) s.found = i;
      }
    }
    __syncthreads();
    p.index = s.found;
    __syncthreads();
    return p;
  }

  // A border in the tokens of a range: `count` of them after n0 of sum sum0.
  __device__ __forceinline__ Place in_range(const Border& b, Range r, uint32_t n0, double sum0, uint32_t count) {
    while (count > (uint32_t)kCap && r.lo < r.hi) {
      // 2^shift keys a bin, at most kBins of them.
      int shift = 0;
      while ((r.hi - r.lo) >> shift >= (uint32_t)kBins) ++shift;
      clear(s.h);
      __syncthreads();
      for_logits<1>(x, 0, V, [&](float v, int) {
        const uint32_t k = key_of(v);
        if (k - r.lo > r.hi - r.lo) return;
        const uint32_t j = (k - r.lo) >> shift;
        atomicAdd(&s.h.count[j], 1u);
        atomicAdd(&s.h.mass[j], fixed(weight(v, m, c), unit));
      });
      __syncthreads();
      const int mine = kBins - 1 - (int)threadIdx.x;
      cumulate(s.h.count[mine], (double)s.h.mass[mine] / unit, n0, sum0);
      const int j = b.by == By::kKey ? kBins - 1 - (int)((b.key - r.lo) >> shift) : bin_with(b);
      n0 = s.count[j];
      sum0 = s.mass[j];
      count = s.count[j + 1] - n0;
      const uint32_t lo = r.lo + ((uint32_t)(kBins - 1 - j) << shift);
      r = Range{lo, min(r.hi, lo + ((1u << shift) - 1))};
      __syncthreads();
    }
    if (count > (uint32_t)kCap) return in_ties(b, r.lo, n0, sum0, count);
    load(r, n0, sum0);
    return in_list(b);
  }
};

// The row's token, from its histogram: this thread's bin (kBins - 1 - thread) has
// count tokens of sum mass.
template <typename T>
__device__ __forceinline__ void select(const SampleArgs& a, int64_t row, float m, double c, bool greedy,
                                       uint32_t count, double mass, Shared& s) {
  const T* const x = static_cast<const T*>(a.x) + row * a.ld;
  if (m == -INFINITY) {   // nothing to choose from
    if (threadIdx.x == 0) {
      a.tokens[row] = -1;
      a.probs[row] = 0.0f;
    }
    return;
  }
  Selector<T> sel{x, a.V, m, c, a.unit, s, Range{1, 0}, 0, 0, 0.0};
  sel.cumulate(count, mass, 0, 0.0);
  const uint32_t all = s.count[kBins];
  const int32_t asked = a.top_k ? a.top_k[row] : a.top_k_all;
  const float top_p = a.top_p ? a.top_p[row] : a.top_p_all, min_p = a.min_p ? a.min_p[row] : a.min_p_all;
  // A top_p of 0 leaves the first one, as a greedy row does.
  const uint32_t k = greedy || top_p <= 0.0f ? 1u : asked > 0 ? min((uint32_t)asked, all) : all;
  const bool by_k = k < all, by_p = !greedy && top_p < 1.0f, by_min = !greedy && min_p > 0.0f;

  // The smallest key of weight min_p: 64 keys of what is left at a time.  Of none
  // above 1.
  uint32_t least = kLowestKey;
  if (by_min) {
    uint32_t lo = kLowestKey - 1, hi = key_of(m) + (min_p > 1.0f);   // hi has the weight, lo has it not
    while (hi - lo > 1) {
      const uint32_t lane = threadIdx.x & 63, span = hi - lo;
      const auto key = [&](uint32_t l) { return lo + (uint32_t)(((u64)span * l + 63) / 64); };
      const u64 yes = __ballot(sel.weight_of(key(lane + 1)) >= (double)min_p);
      const uint32_t first = yes ? (uint32_t)__ffsll((long long)yes) - 1 : 63;
      const uint32_t next = key(first + 1);
      if (first > 0) lo = key(first);
      hi = next;
    }
    least = hi;
  }
  const int bin_min = kBins - 1 - bin_of(least);

  // Which borders there are.  Without both of top-k and top-p, one that is bins
  // below that of min-p does not count.
  int bin_first = kBins - 1;
  if (by_k) bin_first = sel.bin_with(Border{By::kCount, k, 0.0, 0});
  else if (by_p) bin_first = sel.bin_with(Border{By::kSumBelow, 0, top_p * s.mass[kBins], 0});
  const bool min_first = by_min && !(by_k && by_p) && bin_min < bin_first;
  // All that the borders can need, if it is little.
  const int last = min_first ? bin_min : bin_first;
  if (s.count[last + 1] <= (uint32_t)kCap) sel.load(Range{range_of(kBins - 1 - last).lo, kHighestKey}, 0, 0.0);

  uint32_t n = all;
  double sum = s.mass[kBins];
  Place p{};
  for (int step = 0; step < 5; ++step) {
    Border b{};
    if (step == 0) {
      if (!by_k || min_first) continue;
      b = Border{By::kCount, k, 0.0, 0};
    } else if (step == 1) {
      if (!by_p || min_first || n == 1) continue;
      b = Border{By::kSumBelow, 0, (double)top_p * sum, 0};
    } else if (step == 2) {
      if (!by_min || s.count[bin_min] >= n) continue;   // all that is left is above the bin
      b = Border{By::kKey, 0, 0.0, least};
    } else if (step == 3) {
      if (n == 1) continue;
      b = Border{By::kSumAbove, 0, (double)a.u[row] * sum, 0};
    } else {
      if (n > 1 && p.n <= n) continue;
      b = Border{By::kCount, n, 0.0, 0};
    }
    const int j = b.by == By::kKey ? bin_min : sel.bin_with(b);
    const Range r = range_of(kBins - 1 - j);
    // Whatever a border needs is in the list if that holds the border's bin.
    if (sel.held > 0 && r.lo >= sel.range.lo && r.hi <= sel.range.hi) {
      p = sel.in_list(b);
    } else {
      p = sel.in_range(b, r, s.count[j], s.mass[j], s.count[j + 1] - s.count[j]);
      sel.cumulate(count, mass, 0, 0.0);   // the row's bins, where in_range cut one
    }
    if (step < 3 && (p.n < n || step == 0)) {
      n = p.n;
      sum = p.sum;
      if (n < 1) {   // the first one is always kept
        n = 1;
        sum = 1.0;
      }
    }
  }
  if (threadIdx.x == 0) {
    a.tokens[row] = p.index;
    a.probs[row] = (float)(sel.weight_of(p.key) / sum);
  }
}

// A row to a workgroup.
template <typename T>
__global__ void __launch_bounds__(kThreads) sample_kernel(SampleArgs a) {
  __shared__ Shared s;
  for (int64_t row = blockIdx.x; row < a.M; row += gridDim.x) {
    bool greedy;
    const double c = factor(a, row, &greedy);
    const float m = histogram(static_cast<const T*>(a.x) + row * a.ld, 0, a.V, c, a.unit, s.h, s.wave_f);
    const int mine = kBins - 1 - (int)threadIdx.x;
    select<T>(a, row, m, c, greedy, s.h.count[mine], (double)s.h.mass[mine] / a.unit, s);
    __syncthreads();
  }
}

// A part of a row to a workgroup; then a row to a workgroup again.
template <typename T>
__global__ void __launch_bounds__(kThreads) sample_histogram_kernel(SampleArgs a) {
  __shared__ Histogram h;
  __shared__ float part[kWaves];
  const int64_t row = blockIdx.y;
  const int lo = (int)blockIdx.x * a.part, hi = min(lo + a.part, a.V);
  bool greedy;
  const double c = factor(a, row, &greedy);
  const float m = histogram(static_cast<const T*>(a.x) + row * a.ld, lo, hi, c, a.unit, h, part);
  const int64_t at = row * a.splits + blockIdx.x;
  if (threadIdx.x == 0) a.most[at] = m;
  a.mass[at * kBins + threadIdx.x] = h.mass[threadIdx.x];
  a.count[at * kBins + threadIdx.x] = h.count[threadIdx.x];
}

template <typename T>
__global__ void __launch_bounds__(kThreads) sample_select_kernel(SampleArgs a) {
  __shared__ Shared s;
  const int64_t row = blockIdx.x;
  bool greedy;
  const double c = factor(a, row, &greedy);
  float m = -INFINITY;
  for (int i = 0; i < a.splits; ++i) m = fmaxf(m, a.most[row * a.splits + i]);
  uint32_t count = 0;
  double mass = 0.0;
  const int mine = kBins - 1 - (int)threadIdx.x;
  for (int i = 0; i < a.splits; ++i) {
    const int64_t at = row * a.splits + i;
    const float here = a.most[at];
    const uint32_t n = a.count[at * kBins + mine];
    count += n;
    // Each part's sums are relative to its own largest logit.
    if (n) mass += weight(here, m, c) * ((double)a.mass[at * kBins + mine] / a.unit);
  }
  select<T>(a, row, m, c, greedy, count, mass, s);
}

// Parts of a row: a workgroup for each compute unit, of kMinPart logits or more.
int choose_splits(const SampleTokens& c) {
  const int64_t want = device_cus() / c.M, most = ((int64_t)c.V + kMinPart - 1) / kMinPart;
  return (int)(want < 1 ? 1 : want < most ? want : most);
}

template <typename T>
hipError_t launch(const SampleArgs& a, hipStream_t stream) {
  if (a.splits == 1) {
    sample_kernel<T><<<(unsigned)(a.M < 65535 ? a.M : 65535), kThreads, 0, stream>>>(a);
    return hipGetLastError();
  }
  sample_histogram_kernel<T><<<dim3((unsigned)a.splits, (unsigned)a.M), kThreads, 0, stream>>>(a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  sample_select_kernel<T><<<(unsigned)a.M, kThreads, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace

int64_t sample_tokens_workspace(const SampleTokens& c) {
  const int64_t splits = choose_splits(c);
  return splits == 1 ? 0 : c.M * splits * (kBins * 12 + 16);
}

hipError_t launch_sample_tokens(const SampleTokens& c, hipStream_t stream) {
  SampleArgs a{};
  a.x = c.logits;
  a.ld = c.ld;
  a.M = c.M;
  a.V = c.V;
  a.splits = choose_splits(c);
  // Whole cache lines to a part.
  a.part = (int)((((int64_t)c.V + a.splits - 1) / a.splits + 63) / 64 * 64);
  a.splits = (int)(((int64_t)c.V + a.part - 1) / a.part);
  int e = 46;   // the sum of V weights stays below 2^63
  while (((int64_t)c.V >> (63 - e)) != 0) --e;
  a.unit = (double)((int64_t)1 << e);
  a.u = c.uniform;
  a.temperature = c.temperature;
  a.top_p = c.top_p;
  a.min_p = c.min_p;
  a.top_k = c.top_k;
  a.temperature_all = c.temperature_all;
  a.top_p_all = c.top_p_all;
  a.min_p_all = c.min_p_all;
  a.top_k_all = c.top_k_all;
  a.tokens = c.tokens;
  a.probs = c.probs;
  const int64_t parts = c.M * a.splits;
  a.mass = static_cast<u64*>(c.workspace);
  a.count = reinterpret_cast<uint32_t*>(a.mass + parts * kBins);
  a.most = reinterpret_cast<float*>(a.count + parts * kBins);
  return c.fp32 ? launch<float>(a, stream) : launch<__half>(a, stream);
}

}  // namespace dptq
