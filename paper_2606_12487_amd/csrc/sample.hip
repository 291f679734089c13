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
// top-k and top-p mostly leave, they are gathered once for all borders; and with a
// top-p border's bin the bins in which the token's border then lies.  A top-k of up
// to 1024 needs no sums but those of the list: its histogram is of counts alone (256
// x 128256 fp16: 58 -> 42 us; should the list not hold them, the sums are made then).
//
// w in 64 bits: with 131072 tokens of like weight a relative error of 2^-24 in
// the sums would change one token in a hundred.  2^t = 2^n (1 + f q(f)) with n
// the nearest integer and q the interpolant of degree 6 at Chebyshev's nodes on
// [-1/2, 1/2], to 1.2e-10, and alternating, so that sums are closer.
//
// A row to a workgroup where rows are many; few rows are cut into parts whose
// histograms one launch forms, relative to their own largest logit, and a second
// joins.  What bounds it: 256 rows of 100003 fp32 take 56 us, of which the
// histogram is 36 (28 without the weights; some 30 vector instructions a logit,
// 13 of them of 64 bits) and the gathering of the border's bin 13 (a second read
// at 7.8 TB/s).  64 rows of 131072 fp16 that ask for different things take 37 us,
// 12 for the histograms of four parts each and 22 for the second launch on one
// compute unit a row: joining and summing the bins 2.5, gathering 7.5 (13 of two
// ranges), sorting and summing the list 2, and up to four borders in turn, 0.6 each.
// One row of 32000 takes 17 us, the same chain (21 while every wave went through its
// share of a whole span, there or not).  With top-p alone 64 rows of 131072 take 43
// us: two gatherings took 49, at an addition for each vector and not for four.  No
// kernel uses scratch memory: with 92 bytes of it 512 rows of 100003 took 116 us for
// 107.  Dropped, each measured: the gathering shared by a
// row's workgroups, with fences of the device's scope (160 us) or accesses of it
// (56 us: four trips to memory); three loads ahead (registers spill, 39 us); a
// bitonic sort alone (64 rows: 51 us); loops over a chunk's vectors unrolled (the
// code is 50 KB instead of 20 and comes into the instruction cache first: 54 us).
#include "internal.h"
#include "sample_ranges.h"
#include "wave_device.h"

namespace dptq {
namespace {

using namespace sampling;

constexpr int kThreads = 1024, kWaves = kThreads / 64;
static_assert(kBins == kThreads, "a bin a thread");
constexpr int kCap = 2048;        // tokens that are sorted at once
// Parts of a row: logits of each, at least, and how many, at most.
constexpr int kMinPart = 8192, kMaxParts = 8;
constexpr int kXcds = 8;

// a b + c with c in scalar registers: as an FMA of three operands; the compiler
// keeps the constants in vector registers and copies each before its FMA.
__device__ __forceinline__ double fma_scalar(double a, double b, double c) {
  double d;
  asm("v_fma_f64 %0, %1, %2, %3" : "=v"(d) : "v"(a), "v"(b), "s"(c));
  return d;
}

// 2^((x - m) c) in 64 bits, for x <= m; 2^-1000 below that.  (Roundings, conversions
// and scalings of 64 bits run at a quarter of an addition's rate.)
__device__ __forceinline__ double weight(float x, float m, double c) {
  constexpr double kWhole = 0x1.8p52;   // a sum with it is rounded to a whole number, in its low bits
  const double t = fmax(((double)x - (double)m) * c, -1000.0);
  const double s = t + kWhole, f = t - (s - kWhole);
  const int n = __double2loint(s);
  double q = fma_scalar(f, 0x1.00a5814f2a63cp-16, 0x1.443fffcaa2337p-13);
  q = fma_scalar(f, q, 0x1.5d879ead1c114p-10);
  q = fma_scalar(f, q, 0x1.3b2a1b7150c21p-7);
  q = fma_scalar(f, q, 0x1.c6b08d883db58p-5);
  q = fma_scalar(f, q, 0x1.ebfbe045f4d5cp-3);
  q = fma_scalar(f, q, 0x1.62e42fefa39f0p-1);
  q = __builtin_fma(f, q, 1.0);
  return __hiloint2double(__double2hiint(q) + (n << 20), __double2loint(q));   // q 2^n
}

// A weight in units of 2^-e, to the nearest: the sum with 2^52 leaves it in the
// mantissa.  unit = 2^e, e <= 46.
using u64 = unsigned long long;
__device__ __forceinline__ u64 fixed(double w, double unit) {
  return (u64)__double_as_longlong(__builtin_fma(w, unit, 0x1p52)) & 0xFFFFFFFFFFFFFull;
}

// Logits [lo, hi) of a row as a workgroup reads them: what lies before the first
// and after the last whole 16 bytes, a logit to a thread, and between them
// vectors, four to a thread at a time.  The loops over the four are not unrolled:
// the code has to come into the instruction cache first, and a row is not long.
template <typename T>
struct Reader {
  static constexpr int kEach = 16 / sizeof(T), kLoads = 4, kSpan = kLoads * kThreads;
  const T* x;
  int lo, hi, first, vectors;   // first: index of the first vector's first logit
  struct Chunk {
    uint4 v[kLoads];
  };

  __device__ __forceinline__ Reader(const T* row, int from, int to) : x(row), lo(from), hi(to) {
    const int past = (int)((reinterpret_cast<uintptr_t>(x + lo) & 15) / sizeof(T));
    first = min(past ? lo + kEach - past : lo, hi);
    vectors = (hi - first) / kEach;
  }
  __device__ __forceinline__ uint4 none() const {
    const uint32_t w = sizeof(T) == 2 ? 0xFC00FC00u : 0xFF800000u;   // -inf
    return make_uint4(w, w, w, w);
  }
  // Vectors [at, at + kSpan); -inf for those that there are not.
  __device__ __forceinline__ void load(int at, Chunk& c) const {
    const uint4* const p = reinterpret_cast<const uint4*>(x + first);
    if (at + kSpan <= vectors) {
#pragma unroll
      for (int n = 0; n < kLoads; ++n) c.v[n] = p[at + n * kThreads + (int)threadIdx.x];
      return;
    }
#pragma unroll
    for (int n = 0; n < kLoads; ++n) {
      const int i = at + n * kThreads + (int)threadIdx.x;
      c.v[n] = none();
      if (i < vectors) c.v[n] = p[i];
    }
  }
  // Whether this wave has any of the n-th vectors of the span at `at`.
  __device__ __forceinline__ bool any(int at, int n) const {
    return at + n * kThreads + __builtin_amdgcn_readfirstlane((int)threadIdx.x & ~63) < vectors;
  }
  // f(logit, number in its vector, index of the vector's first logit), vector by vector.
  template <typename F>
  __device__ __forceinline__ void each(Chunk c, int at, const F& f) const {
    int i = first + (at + (int)threadIdx.x) * kEach;
#pragma unroll 1
    for (int n = 0; n < kLoads && any(at, n); ++n) {
      f(c.v[0], i);
#pragma unroll
      for (int k = 0; k + 1 < kLoads; ++k) c.v[k] = c.v[k + 1];
      i += kThreads * kEach;
    }
  }
  // The thread's logit of the ends, as a vector of it and -inf, and its index.
  __device__ __forceinline__ uint4 ends(int& i) const {
    const int t = threadIdx.x, last = first + vectors * kEach;
    i = t < first - lo ? lo + t : t >= 64 && t - 64 < hi - last ? last + t - 64 : -1;
    uint4 v = none();
    if (i >= 0) {
      if constexpr (sizeof(T) == 2) v.x = 0xFC000000u | __half_as_ushort(x[i]);
      else v.x = __float_as_uint(x[i]);
    }
    return v;
  }
};
template <typename T, typename F>
__device__ __forceinline__ void values(uint4 v, const F& f) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    if constexpr (sizeof(T) == 2) {
      const __half2 h = *reinterpret_cast<const __half2*>(&w[k]);
      f(__low2float(h), 2 * k);
      f(__high2float(h), 2 * k + 1);
    } else {
      f(__uint_as_float(w[k]), k);
    }
  }
}

// A value that all lanes have, in a scalar register.
__device__ __forceinline__ uint32_t scalar(uint32_t x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ u64 scalar(u64 x) {
  return (u64)scalar((uint32_t)(x >> 32)) << 32 | scalar((uint32_t)x);
}

// Which values of a vector lie in a range, as bits; element(b): which value a bit
// is.  NaN does not; -0 is 0.
template <typename T>
struct Within {
  float least, most;
  __device__ __forceinline__ explicit Within(Range r) : least(value_of(r.lo)), most(value_of(r.hi)) {}
  __device__ __forceinline__ uint32_t marks(uint4 v) const {
    uint32_t m = 0;
    values<T>(v, [&](float e, int j) { m |= e >= least && e <= most ? 1u << j : 0u; });
    return m;
  }
  __device__ __forceinline__ static int element(int b) { return b & 3; }
};
// fp16: two at a time, those that clamping to the range's least and most fp16
// number leaves as they are; none where no number lies in the range, as clamping
// leaves `most` as it is there.
template <>
struct Within<__half> {
  typedef _Float16 half2_t __attribute__((ext_vector_type(2)));
  typedef unsigned short ushort2_t __attribute__((ext_vector_type(2)));
  half2_t least, most;
  uint32_t all;   // the bits of a vector's values
  __device__ __forceinline__ explicit Within(Range r) {
    const HalfRange in = halves_of(Range{scalar(r.lo), scalar(r.hi)});
    const unsigned short l = half_bits(in.least), h = half_bits(in.most);
    const ushort2_t a = {l, l}, b = {h, h};
    all = in.least <= in.most ? 0x000F000Fu : 0;
    least = __builtin_bit_cast(half2_t, a);
    most = __builtin_bit_cast(half2_t, b);
  }
  __device__ __forceinline__ uint32_t marks(uint4 v) const {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    const ushort2_t one = {1, 1};
    uint32_t out = 0;   // bits k and 16 + k: the values of dword k lie outside
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const half2_t e = __builtin_bit_cast(half2_t, w[k]) + (half2_t)(_Float16)0;
      const half2_t c = __builtin_elementwise_min(__builtin_elementwise_max(e, least), most);
      const ushort2_t d = __builtin_bit_cast(ushort2_t, __builtin_bit_cast(uint32_t, c) ^ __builtin_bit_cast(uint32_t, e));
      out |= __builtin_bit_cast(uint32_t, __builtin_elementwise_min(d, one)) << k;
    }
    return ~out & all;
  }
  __device__ __forceinline__ static int element(int b) { return 2 * (b & 3) + (b >> 4); }
};

struct SampleArgs {
  const void* x;
  int64_t ld, M;
  int V, splits, part;      // part: logits of a split
  double unit;              // 2^e of the sums of a row
  u64 one;                  // the same
  const float* u;
  const float *temperature, *top_p, *min_p;   // of each row, or nullptr and the value
  const int32_t* top_k;
  float temperature_all, top_p_all, min_p_all;
  int top_k_all;
  int64_t* tokens;
  float* probs;
  // Of rows in parts, from the first launch: their histograms.
  u64* mass;                // [M][splits][kBins]
  uint32_t* count;
  float* most;              // [M][splits]
};

// What a row asks for.
struct Asked {
  double c;        // log2(e) / T; a greedy row (T = 0) is that of T = 1
  float u, top_p, min_p;
  uint32_t top_k;  // 0: all
  bool greedy;
  // Whether the row's sums are needed: not where the list will hold the top_k
  // tokens, and with them all that is asked for.
  bool sums;
};
__device__ __forceinline__ Asked asked_of(const SampleArgs& a, int64_t row) {
  const float t = a.temperature ? a.temperature[row] : a.temperature_all;
  const int32_t k = a.top_k ? a.top_k[row] : a.top_k_all;
  Asked q;
  q.u = a.u[row];
  q.top_p = a.top_p ? a.top_p[row] : a.top_p_all;
  q.min_p = a.min_p ? a.min_p[row] : a.min_p_all;
  q.greedy = !(t > 0.0f);
  q.c = 1.4426950408889634 / (q.greedy ? 1.0 : (double)t);
  // A top_p of 0 or a min_p above 1 leaves the first one, as a greedy row does.
  q.top_k = q.greedy || q.top_p <= 0.0f || q.min_p > 1.0f ? 1u : k > 0 ? (uint32_t)k : 0u;
  q.sums = q.top_k == 0 || q.top_k > (uint32_t)kCap / 2;
  return q;
}

struct Histogram {
  u64 mass[kBins];
  uint32_t count[kBins];
};

// All tokens of a range, in the list.
struct Segment {
  Range range;
  uint32_t first, held;   // in the list
  uint32_t before_n;      // tokens of the row before it
  u64 before_sum;
};

struct Shared {
  Histogram h;                 // of the row, then of a bin that is cut again
  u64 mass[kBins + 1];         // before bin kBins - 1 - j
  uint32_t count[kBins + 1];
  u64 list[kCap];              // key and ~index, in the order
  u64 sum[kCap];               // up to each
  Segment seg[2];              // what the list holds: a range, or two, the second before the first
  u64 wave_m[2][kWaves];
  uint32_t wave_n[2][kWaves];
  float wave_f[2][kWaves];
  int n, found;
};

// The sum of the waves before this one, of each wave's value (lane 63's), in
// part; a barrier comes before the reads, and the callers alternate between two
// parts.
template <typename V>
__device__ __forceinline__ void put_wave(V x, V* part) {
  if ((threadIdx.x & 63) == 63) part[threadIdx.x >> 6] = x;
}
template <typename V>
__device__ __forceinline__ V waves_before(const V* part) {
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const V x = wave_scan((threadIdx.x & 63) < kWaves ? part[threadIdx.x & 63] : (V)0);
  V before = 0;
  if constexpr (sizeof(V) == 8) {
    const uint32_t lo = __builtin_amdgcn_readlane((uint32_t)x, wave ? wave - 1 : 0);
    const uint32_t hi = __builtin_amdgcn_readlane((uint32_t)(x >> 32), wave ? wave - 1 : 0);
    before = (u64)hi << 32 | lo;
  } else {
    before = __builtin_amdgcn_readlane(x, wave ? wave - 1 : 0);
  }
  return wave ? before : (V)0;
}

// The histogram of logits [lo, hi) of a row, relative to the largest of them,
// which it returns: chunk by chunk, and where a larger one comes up the sums so
// far are scaled down to it.  Without `sums` these stay 0.  Barriers: none at the
// end.
template <typename T>
__device__ __forceinline__ float histogram(const T* x, int lo, int hi, double c, double unit, bool sums, Histogram& h,
                                           float (*part)[kWaves]) {
  using R = Reader<T>;
  const int tid = threadIdx.x;
  h.mass[tid] = 0;
  h.count[tid] = 0;
  const R r(x, lo, hi);
  typename R::Chunk now, next;
  r.load(0, now);
  int unused;
  const uint4 ends = r.ends(unused);
  float m = -INFINITY;
  int parity = 0;
  for (int at = 0; at < r.vectors || at == 0; at += R::kSpan) {
    if (at + R::kSpan < r.vectors) r.load(at + R::kSpan, next);
    float most = -INFINITY;
    const auto larger = [&](float v, int) { most = fmaxf(most, v); };
#pragma unroll
    for (int n = 0; n < R::kLoads; ++n) values<T>(now.v[n], larger);
    if (at == 0) values<T>(ends, larger);
    most = wave_max(most);
    put_wave(most, part[parity]);
    __syncthreads();   // and the last chunk's sums are there
    most = wave_max(part[parity][tid & (kWaves - 1)]);
    parity ^= 1;
    if (most > m) {
      if (m > -INFINITY) h.mass[tid] = __double2ull_rn((double)h.mass[tid] * weight(m, most, c));
      m = most;
      __syncthreads();
    }
    if (most > -INFINITY) {
      const auto add = [&](float v, int) {
        const int b = bin_of(v);
        const u64 w = fixed(weight(v, m, c), unit);
        if (!(v > -INFINITY)) return;   // masked, or NaN
        atomicAdd(&h.count[b], 1u);
        atomicAdd(&h.mass[b], w);
      };
      const auto count = [&](float v, int) {
        if (v > -INFINITY) atomicAdd(&h.count[bin_of(v)], 1u);
      };
      if (sums) r.each(now, at, [&](uint4 v, int) { values<T>(v, add); });
      else r.each(now, at, [&](uint4 v, int) { values<T>(v, count); });
      if (at == 0 && (lo < r.first || hi > r.first + r.vectors * R::kEach)) {
        // The ends' single logits.
        float v;
        if constexpr (sizeof(T) == 2) v = __half2float(__ushort_as_half((unsigned short)ends.x));
        else v = __uint_as_float(ends.x);
        if (sums) add(v, 0);
        else count(v, 0);
      }
    }
    now = next;
  }
  return m;
}

// What a border is given by.
enum class By { kCount, kSum, kKey };
struct Border {
  By by;
  uint32_t n;      // kCount: the n-th token is the last before it (n >= 1)
  u64 sum;         // kSum: the first token up to which the sum is this or more is
                   // the last before it (sum > 0)
  uint32_t key;    // kKey: it stands behind the tokens of this key and above
};
// Where it is: tokens before it, their sum, and the last of them.
struct Place {
  uint32_t n;
  u64 sum;
  uint32_t key;
  int index;
};

// The first of `size` that holds, of a condition that holds for all behind it
// too; size (a power of two, at most 64 * 64) if none does.  By every wave for
// itself.
template <typename F>
__device__ __forceinline__ int first_of(int size, const F& holds) {
  const int lane = threadIdx.x & 63;
  int at = 0;
  if (size > 64) {
    const int step = size / 64;
    const u64 yes = __ballot(holds(step * lane + step - 1));
    if (!yes) return size;
    at = step * (__ffsll((long long)yes) - 1);
    size = step;
  }
  const u64 yes = __ballot(lane < size && holds(at + (lane < size ? lane : 0)));
  return yes ? at + __ffsll((long long)yes) - 1 : at + size;
}

// One stage of a bitonic sort of size keys in the order (largest first), e of a
// thread: key p = 1024 e + thread meets key p ^ j.
__device__ __forceinline__ u64 better(u64 mine, u64 other, bool first) {
  return (mine > other) == first ? mine : other;
}
template <int J>
__device__ __forceinline__ u64 lane_xor64(u64 x) {
  return (u64)lane_xor<J>((uint32_t)(x >> 32)) << 32 | lane_xor<J>((uint32_t)x);
}
template <int J>
__device__ __forceinline__ void sort_in_wave(u64& v, uint32_t p, uint32_t k) {
  v = better(v, lane_xor64<J>(v), ((p & J) == 0) == ((p & k) == 0));
}
__device__ __forceinline__ void sort_list(u64* list, int size) {
  const uint32_t tid = threadIdx.x;
  constexpr int E = kCap / kThreads;
  u64 v[E];
  bool mine[E];   // of whole waves
#pragma unroll
  for (int e = 0; e < E; ++e) {
    mine[e] = (int)(e * kThreads + tid) < size;
    v[e] = mine[e] ? list[e * kThreads + tid] : 0;
  }
  __syncthreads();
  for (uint32_t k = 2; k <= (uint32_t)size; k *= 2) {
    for (uint32_t j = k / 2; j >= 64; j /= 2) {
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (mine[e]) list[e * kThreads + tid] = v[e];
      __syncthreads();
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const uint32_t p = e * kThreads + tid;
        if (mine[e]) v[e] = better(v[e], list[p ^ j], ((p & j) == 0) == ((p & k) == 0));
      }
      __syncthreads();
    }
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const uint32_t p = e * kThreads + tid;
      if (!mine[e]) continue;
      if (k >= 64) sort_in_wave<32>(v[e], p, k);
      if (k >= 32) sort_in_wave<16>(v[e], p, k);
      if (k >= 16) sort_in_wave<8>(v[e], p, k);
      if (k >= 8) sort_in_wave<4>(v[e], p, k);
      if (k >= 4) sort_in_wave<2>(v[e], p, k);
      sort_in_wave<1>(v[e], p, k);
    }
  }
#pragma unroll
  for (int e = 0; e < E; ++e)
    if (mine[e]) list[e * kThreads + tid] = v[e];
  __syncthreads();
}

template <typename T>
struct Selector {
  const T* x;
  int V;
  float m;
  double c, unit;
  Shared& s;

  // Tokens of a range of keys: `count` of them after n0 of sum sum0.
  struct Part {
    Range r;
    uint32_t n0, count;
    u64 sum0;
  };

  __device__ __forceinline__ double weight_of(uint32_t key) const { return weight(value_of(key), m, c); }

  // The cumulative counts and sums of bins, descending (this thread's is the one
  // after those of lower threads), after n tokens of sum `sum`.
  __device__ __forceinline__ void cumulate(uint32_t count, u64 mass, uint32_t n, u64 sum, uint32_t* counts,
                                           u64* sums) {
    const uint32_t cn = wave_scan(count);
    const u64 cm = wave_scan(mass);
    put_wave(cn, s.wave_n[0]);
    put_wave(cm, s.wave_m[0]);
    __syncthreads();
    counts[threadIdx.x + 1] = n + waves_before(s.wave_n[0]) + cn;
    sums[threadIdx.x + 1] = sum + waves_before(s.wave_m[0]) + cm;
    if (threadIdx.x == 0) counts[0] = n, sums[0] = sum;
    __syncthreads();
  }

  // Which of the cumulated bins (0: the first in the order) a border is in; the
  // last that is not empty where rounding leaves none.  kKey does not come here.
  __device__ __forceinline__ int bin_with(const Border& b, const uint32_t* counts, const u64* sums) const {
    int j = kBins;
    if (b.by == By::kSum) j = first_of(kBins, [&](int i) { return sums[i + 1] >= b.sum; });
    if (j == kBins) {
      const uint32_t n = b.by == By::kCount ? b.n : counts[kBins];
      j = first_of(kBins, [&](int i) { return counts[i + 1] >= n; });
    }
    return min(j, kBins - 1);
  }
  // Of the row's.
  __device__ __forceinline__ int bin_with(const Border& b) const { return bin_with(b, s.count, s.mass); }

  // The tokens of bins j to k of the row's.
  __device__ __forceinline__ Part bins(int j, int k) const {
    const uint32_t n0 = scalar(s.count[j]);
    return {Range{range_of(kBins - 1 - k).lo, range_of(kBins - 1 - j).hi}, n0, scalar(s.count[k + 1]) - n0,
            scalar(s.mass[j])};
  }

  // Gathers the tokens of a range, or of two, into the list, in any order; their
  // number, at most kCap.
  __device__ __forceinline__ int gather(Range r, bool two, Range r2) {
    __syncthreads();   // the list's readers are done
    if (threadIdx.x == 0) s.n = 0;
    __syncthreads();
    const Within<T> within(r), within2(r2);
    using R = Reader<T>;
    // The row's address is made anew: the compiler would keep those of all loads over
    // the selection's steps, and spill others for them.
    const T* row = x;
    asm volatile("" : "+s"(row));
    const R reader(row, 0, V);
    // A thread marks what it has of up to four vectors, index_of(bit) the first bit's
    // logit and so on, and puts down the indices.
    const auto marks = [&](uint4 v) {
      uint32_t mine = within.marks(v);
      if (two) mine |= within2.marks(v);
      return mine;
    };
    const auto put = [&](uint32_t mine, const auto& index_of) {
      if (!mine) return;
      // One addition for each lane as it is: the compiler would sum up a uniform
      // address's over the wave, which takes longer for the few lanes here.
      int offset;
      asm("v_mov_b32 %0, 0" : "=v"(offset));
      int to = atomicAdd(&s.n + offset, __popc(mine));
      for (; mine; mine &= mine - 1, ++to)
        if (to < kCap) s.list[to] = (u64)index_of(__ffs((int)mine) - 1);
    };
    const auto take = [&](const typename R::Chunk& c, int at) {
      uint32_t mine = 0;
#pragma unroll
      for (int n = 0; n < R::kLoads; ++n) mine |= marks(c.v[n]) << (4 * n);
      const int i = reader.first + (at + (int)threadIdx.x) * R::kEach;
      put(mine, [&](int b) { return i + (b >> 2 & 3) * kThreads * R::kEach + Within<T>::element(b); });
    };
    typename R::Chunk even, odd;   // one on its way while the other is taken
    int i;
    const uint4 ends = reader.ends(i);
    reader.load(0, even);
    put(marks(ends), [&](int) { return i; });
    for (int at = 0; at < reader.vectors; at += 2 * R::kSpan) {
      const int next = at + R::kSpan;
      if (next < reader.vectors) reader.load(next, odd);
      take(even, at);
      if (next >= reader.vectors) break;
      if (next + R::kSpan < reader.vectors) reader.load(next + R::kSpan, even);
      take(odd, next);
    }
    __syncthreads();
    const int count = min((int)scalar((uint32_t)s.n), kCap);
    for (int k = threadIdx.x; k < count; k += kThreads) {
      const uint32_t at = (uint32_t)s.list[k];   // V < 2^30: 32 bits of bytes
      const T v = *reinterpret_cast<const T*>(reinterpret_cast<const char*>(row) + at * (uint32_t)sizeof(T));
      s.list[k] = (u64)key_of((float)v) << 32 | ~at;
    }
    return count;
  }

  // Sorts the list's tokens: counted into kBins stretches of the range (without the
  // `gap` keys below `split`), scattered to their stretch, and each put behind those
  // of it that come first.  A stretch holds a few; false, and nothing done, where one
  // holds more than kCrowd.
  __device__ __forceinline__ bool sort_by_buckets(int count, Range r, uint32_t split, uint32_t gap) {
    constexpr int E = kCap / kThreads, kCrowd = 64;
    uint32_t* const offset = reinterpret_cast<uint32_t*>(s.h.mass);   // [kBins + 1]
    const int tid = threadIdx.x;
    const Buckets buckets = buckets_of(r, split, gap);
    s.h.count[tid] = 0;
    if (tid == 0) s.found = 0;
    __syncthreads();
    u64 v[E];
    uint32_t bucket[E], place[E];
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int i = e * kThreads + tid;
      if (i >= count) continue;
      v[e] = s.list[i];
      bucket[e] = bucket_of(buckets, (uint32_t)(v[e] >> 32));
      place[e] = atomicAdd(&s.h.count[bucket[e]], 1u);
      if (place[e] >= (uint32_t)kCrowd) s.found = 1;
    }
    __syncthreads();
    if (s.found) return false;
    const uint32_t mine = s.h.count[tid], up_to = wave_scan(mine);
    put_wave(up_to, s.wave_n[1]);
    __syncthreads();
    const uint32_t end = waves_before(s.wave_n[1]) + up_to;
    offset[tid + 1] = end;
    if (tid == 0) offset[0] = 0;
    __syncthreads();
#pragma unroll
    for (int e = 0; e < E; ++e)
      if (e * kThreads + tid < count) s.sum[offset[bucket[e]] + place[e]] = v[e];
    __syncthreads();
#pragma unroll
    for (int e = 0; e < E; ++e) {
      if (e * kThreads + tid >= count) continue;
      const uint32_t from = offset[bucket[e]], to = offset[bucket[e] + 1];
      uint32_t at = from;
      for (uint32_t i = from; i < to; ++i) at += s.sum[i] > v[e];
      s.list[at] = v[e];
    }
    __syncthreads();
    return true;
  }

  // Puts `count` gathered tokens in their order, with their sums: all of the part,
  // or, `ahead` holding any, of that one too.
  __device__ __forceinline__ void arrange(int count, const Part& part, const Part& ahead) {
    const bool two = ahead.count > 0;
    const Range r{part.r.lo, two ? ahead.r.hi : part.r.hi};
    if (!sort_by_buckets(count, r, two ? ahead.r.lo : 0, two ? ahead.r.lo - part.r.hi - 1 : 0)) {
      int size = 64;
      while (size < count) size *= 2;
      for (int i = count + threadIdx.x; i < size; i += kThreads) s.list[i] = 0;   // behind all
      __syncthreads();
      sort_list(s.list, size);
    }
    const int a = 2 * threadIdx.x;
    const u64 w0 = a < count ? fixed(weight_of((uint32_t)(s.list[a] >> 32)), unit) : 0;
    const u64 w1 = a + 1 < count ? fixed(weight_of((uint32_t)(s.list[a + 1] >> 32)), unit) : 0;
    const u64 up_to = wave_scan(w0 + w1);
    put_wave(up_to, s.wave_m[1]);
    __syncthreads();
    const u64 all = waves_before(s.wave_m[1]) + up_to;
    s.sum[a] = all - w1;
    s.sum[a + 1] = all;
    if (threadIdx.x == 0) {
      const uint32_t first = min(ahead.count, (uint32_t)count);
      s.seg[0] = Segment{part.r, first, (uint32_t)count - first, part.n0, part.sum0};
      s.seg[1] = Segment{ahead.r, 0, first, ahead.n0, ahead.sum0};
    }
    __syncthreads();
  }

  // The segment that holds all of a range; -1: none.
  __device__ __forceinline__ int holder(Range r) const {
#pragma unroll
    for (int i = 0; i < 2; ++i)
      if (s.seg[i].held > 0 && r.lo >= s.seg[i].range.lo && r.hi <= s.seg[i].range.hi) return i;
    return -1;
  }

  // A border among a segment's tokens.
  __device__ __forceinline__ Place in_list(const Border& b, int held) const {
    const Segment& in = s.seg[held];
    const struct {
      uint32_t first, held, before_n;
      u64 before_sum;
    } g{scalar(in.first), scalar(in.held), scalar(in.before_n), scalar(in.before_sum)};
    const int first = (int)g.first, end = (int)(g.first + g.held);
    const u64 base = first ? scalar(s.sum[first - 1]) : 0;
    uint32_t n;   // tokens of it before the border
    if (b.by == By::kCount) {
      n = b.n - g.before_n;
    } else if (b.by == By::kKey) {
      n = first_of(kCap, [&](int i) { return i >= end || (i >= first && (uint32_t)(s.list[i] >> 32) < b.key); }) - first;
    } else {
      const u64 least = b.sum - min(b.sum, g.before_sum) + base;
      n = 1 + first_of(kCap, [&](int i) { return i >= end || (i >= first && s.sum[i] >= least); }) - first;
    }
    n = min(n, g.held);
    Place p{g.before_n + n, g.before_sum, 0, -1};
    if (n) {
      const u64 last = scalar(s.list[first + n - 1]);
      p.sum = g.before_sum + (scalar(s.sum[first + n - 1]) - base);
      p.key = (uint32_t)(last >> 32);
      p.index = (int)~(uint32_t)last;
    }
    return p;
  }

  // A border among `count` equal values.
  __device__ __forceinline__ Place in_ties(const Border& b, uint32_t key, uint32_t n0, u64 sum0, uint32_t count) {
    const u64 w = fixed(weight_of(key), unit);
    uint32_t k = count;
    if (b.by == By::kCount) k = min(b.n - n0, count);
    else if (b.by == By::kKey) k = key >= b.key ? count : 0;
    else if (w) k = (uint32_t)min((b.sum - min(b.sum, sum0) + w - 1) / w, (u64)count);
    Place p{n0 + k, sum0 + k * w, key, -1};
    if (k == 0) return p;
    // The k-th of them by index: each thread counts those of a stretch.
    const int stretch = (V + kThreads - 1) / kThreads;
    const int lo = (int)min((int64_t)threadIdx.x * stretch, (int64_t)V), hi = min(lo + stretch, V);
    uint32_t mine = 0;
    for (int i = lo; i < hi; ++i) mine += key_of((float)x[i]) == key;
    uint32_t up_to = wave_scan(mine);
    put_wave(up_to, s.wave_n[1]);
    if (threadIdx.x == 0) s.found = -1;
    __syncthreads();
    up_to += waves_before(s.wave_n[1]);
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

  // The part of a range with more than kCap tokens that a border is in: at most
  // kCap, or all equal.  The list's memory holds the bins' sums meanwhile, so the
  // list is empty.
  __device__ __forceinline__ Part narrow(const Border& b, Part p) {
    uint32_t* const counts = reinterpret_cast<uint32_t*>(s.list);
    u64* const sums = s.sum;
    static_assert(kCap > kBins, "the bins' sums in the list");
    while (p.count > (uint32_t)kCap && p.r.lo < p.r.hi) {
      // 2^shift keys a bin, at most kBins of them.
      int shift = 0;
      while ((p.r.hi - p.r.lo) >> shift >= (uint32_t)kBins) ++shift;
      s.h.mass[threadIdx.x] = 0;
      s.h.count[threadIdx.x] = 0;
      __syncthreads();
      if (threadIdx.x < 2) s.seg[threadIdx.x].held = 0;
      for (int i = threadIdx.x; i < V; i += kThreads) {
        const float v = (float)x[i];
        const uint32_t k = key_of(v);
        if (k - p.r.lo > p.r.hi - p.r.lo) continue;
        const uint32_t j = (k - p.r.lo) >> shift;
        atomicAdd(&s.h.count[j], 1u);
        atomicAdd(&s.h.mass[j], fixed(weight(v, m, c), unit));
      }
      __syncthreads();
      const int mine = kBins - 1 - (int)threadIdx.x;
      cumulate(s.h.count[mine], s.h.mass[mine], p.n0, p.sum0, counts, sums);
      const int j = b.by == By::kKey ? kBins - 1 - (int)((b.key - p.r.lo) >> shift) : bin_with(b, counts, sums);
      p.n0 = scalar(counts[j]);
      p.sum0 = scalar(sums[j]);
      p.count = scalar(counts[j + 1]) - p.n0;
      const uint32_t lo = p.r.lo + ((uint32_t)(kBins - 1 - j) << shift);
      p.r = Range{lo, min(p.r.hi, lo + ((1u << shift) - 1))};
      __syncthreads();
    }
    return p;
  }
};

// The least sum that is not below p of `sum`, and the least that is above u of it.
// (The empty asm keeps the conversion of p or u here: the compiler would make them
// ahead of the selection's steps, and spill them.)
__device__ __forceinline__ double wide(float p) {
  asm volatile("" : "+s"(p));
  return (double)p;
}
__device__ __forceinline__ u64 below(float p, u64 sum) { return max(__double2ull_ru(wide(p) * (double)sum), 1ull); }
__device__ __forceinline__ u64 above(float u, u64 sum) {
  return __double2ull_rd(fmax(wide(u) * (double)sum, 0.0)) + 1;
}

// The row's token, from its histogram: this thread's bin (kBins - 1 - thread) has
// count tokens of sum mass.
template <typename T>
__device__ __forceinline__ void select(const SampleArgs& a, int64_t row, float m, const Asked& asked, uint32_t count,
                                       u64 mass, Shared& s) {
  const T* const x = static_cast<const T*>(a.x) + row * a.ld;
  if (m == -INFINITY) {   // nothing to choose from
    if (threadIdx.x == 0) {
      a.tokens[row] = -1;
      a.probs[row] = 0.0f;
    }
    return;
  }
  m = __uint_as_float(scalar(__float_as_uint(m)));
  Selector<T> sel{x, a.V, m, asked.c, a.unit, s};
  if (threadIdx.x < 2) s.seg[threadIdx.x].held = 0;
  sel.cumulate(count, mass, 0, 0, s.count, s.mass);
  const uint32_t all = scalar(s.count[kBins]);
  const float top_p = asked.top_p, min_p = asked.min_p;
  const uint32_t k = asked.top_k ? min(asked.top_k, all) : all;
  const bool by_k = k < all, by_p = !asked.greedy && top_p < 1.0f && k > 1;
  const bool by_min = !asked.greedy && min_p > 0.0f && k > 1;

  // The smallest key of weight min_p: 64 keys of what is left at a time.
  uint32_t least = kLowestKey;
  if (by_min) {
    uint32_t lo = kLowestKey - 1, hi = key_of(m);   // hi has the weight, lo has it not
    while (hi - lo > 1) {
      const uint32_t lane = threadIdx.x & 63, span = hi - lo;
      const auto key = [&](uint32_t l) { return lo + (span >> 6) * l + (((span & 63) * l + 63) >> 6); };   // + span l / 64
      const u64 yes = __ballot(sel.weight_of(key(lane + 1)) >= (double)min_p);
      const uint32_t first = yes ? (uint32_t)__ffsll((long long)yes) - 1 : 63;
      const uint32_t next = key(first + 1);
      if (first > 0) lo = key(first);
      hi = next;
    }
    least = key_of(value_of(hi));   // -0 is 0
  }
  const int bin_min = kBins - 1 - bin_of(least);

  // Which borders there are.  Without both of top-k and top-p, one that is bins
  // below that of min-p does not count.  (Without the sums a border by one is behind
  // the last token here: a row of at most top_k tokens, all in the list.)
  int bin_first = kBins - 1;
  if (by_k) bin_first = sel.bin_with(Border{By::kCount, k, 0, 0});
  else if (by_p) bin_first = sel.bin_with(Border{By::kSum, 0, below(top_p, s.mass[kBins]), 0});
  const bool min_first = by_min && (by_k ? !by_p : asked.sums) && bin_min < bin_first;
  const int last = min_first ? bin_min : bin_first;

  if (!asked.sums && s.count[last + 1] > (uint32_t)kCap) {
    // More tokens in the bin than expected: the sums after all.
    s.h.mass[threadIdx.x] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < a.V; i += kThreads) {
      const float v = (float)x[i];
      if (v > -INFINITY) atomicAdd(&s.h.mass[bin_of(v)], fixed(weight(v, m, asked.c), a.unit));
    }
    __syncthreads();
    sel.cumulate(count, s.h.mass[kBins - 1 - (int)threadIdx.x], 0, 0, s.count, s.mass);
  }

  uint32_t n = all;
  u64 sum = scalar(s.mass[kBins]);
  Place p{};
  bool whole = false;   // the list has all
  for (int step = -1; step < 5; ++step) {
    Border b{};
    typename Selector<T>::Part part{}, ahead{};
    int held = -1;
    bool placed = false;
    if (step < 0) {
      // All that the borders can need, if it is little.
      part = {Range{range_of(kBins - 1 - last).lo, key_of(m)}, 0, scalar(s.count[last + 1]), 0};
      if (part.count > (uint32_t)kCap) continue;
      whole = true;
    } else {
      if (step == 0) {
        if (!by_k || min_first) continue;
        b = Border{By::kCount, k, 0, 0};
      } else if (step == 1) {
        if (!by_p || min_first || n == 1) continue;
        b = Border{By::kSum, 0, below(top_p, sum), 0};
      } else if (step == 2) {
        if (!by_min || s.count[bin_min] >= n) continue;   // all that is left is above the bin
        b = Border{By::kKey, 0, 0, least};
      } else if (step == 3) {
        if (n == 1) continue;
        b = Border{By::kSum, 0, above(asked.u, sum), 0};
      } else {
        if (n > 1 && p.n <= n) continue;
        b = Border{By::kCount, n, 0, 0};
      }
      if (whole) {
        held = 0;
      } else {
        const int j = b.by == By::kKey ? bin_min : sel.bin_with(b);
        part = sel.bins(j, j);
        // Whatever a border needs is in the list if that holds the border's bin.
        held = sel.holder(part.r);
        if (held < 0 && step == 1 && !by_min) {
          // The token's border is in one of these bins, wherever in bin j this one
          // turns out to be: gathered with it where both are little.
          const int from = sel.bin_with(Border{By::kSum, 0, above(asked.u, s.mass[j]), 0});
          const int to = sel.bin_with(Border{By::kSum, 0, above(asked.u, s.mass[j + 1]), 0});
          if (s.count[min(to, j) + 1] - s.count[from] + part.count <= (uint32_t)kCap) {
            if (to < j) ahead = sel.bins(from, to);
            else part = sel.bins(min(from, j), j);
          }
        }
      }
      if (held < 0 && part.count > (uint32_t)kCap) {
        part = sel.narrow(b, part);
        placed = part.count > (uint32_t)kCap;
        if (placed) p = sel.in_ties(b, part.r.lo, part.n0, part.sum0, part.count);
      }
      // No token in a border's range (a min-p border's, and most stretches of one that
      // is cut are empty): it stands behind those before the range.
      if (held < 0 && part.count == 0) {
        placed = true;
        p = Place{part.n0, part.sum0, 0, -1};
      }
    }
    if (held < 0 && !placed) {
      sel.arrange(sel.gather(part.r, ahead.count > 0, ahead.r), part, ahead);
      held = 0;
    }
    if (step < 0) {
      if (part.count == all) sum = scalar(s.sum[all - 1]);
      continue;
    }
    if (!placed) p = sel.in_list(b, held);
    if (step < 3 && (p.n < n || step == 0)) {
      n = p.n;
      sum = p.sum;
      if (n < 1) {   // the first one is always kept
        n = 1;
        sum = a.one;
      }
    }
  }
  if (threadIdx.x == 0) {
    a.tokens[row] = p.index;
    a.probs[row] = (float)(sel.weight_of(p.key) * a.unit / (double)sum);
  }
}

// A row to a workgroup, from row `first`.
template <typename T>
__global__ void __launch_bounds__(kThreads) sample_kernel(SampleArgs a, int64_t first) {
  __shared__ Shared s;
  const int64_t row = first + blockIdx.x;
  const Asked asked = asked_of(a, row);
  const float m =
      histogram(static_cast<const T*>(a.x) + row * a.ld, 0, a.V, asked.c, a.unit, asked.sums, s.h, s.wave_f);
  __syncthreads();
  const int mine = kBins - 1 - (int)threadIdx.x;
  select<T>(a, row, m, asked, s.h.count[mine], s.h.mass[mine], s);
}

// A part of a row to a workgroup; then a row to a workgroup again.
template <typename T>
__global__ void __launch_bounds__(kThreads) sample_histogram_kernel(SampleArgs a) {
  __shared__ Histogram h;
  __shared__ float part[2][kWaves];
  // A row's parts on the XCD (workgroup mod 8) that its second launch runs on,
  // whose L2 then has their histograms and the row (64 rows of 131072 in four
  // parts: 12 us for 13, and the second launch reads them in 1.3 us for 1.9).
  const int turn = (int)blockIdx.x / kXcds, split = turn % a.splits;
  const int64_t row = (int64_t)(turn / a.splits) * kXcds + blockIdx.x % kXcds;
  if (row >= a.M) return;
  const int lo = split * a.part, hi = min(lo + a.part, a.V);
  const Asked asked = asked_of(a, row);
  const float m = histogram(static_cast<const T*>(a.x) + row * a.ld, lo, hi, asked.c, a.unit, asked.sums, h, part);
  __syncthreads();
  const int64_t at = row * a.splits + split;
  if (threadIdx.x == 0) a.most[at] = m;
  a.mass[at * kBins + threadIdx.x] = h.mass[threadIdx.x];
  a.count[at * kBins + threadIdx.x] = h.count[threadIdx.x];
}

template <typename T>
__global__ void __launch_bounds__(kThreads) sample_select_kernel(SampleArgs a) {
  __shared__ Shared s;
  const int64_t row = blockIdx.x;
  const Asked asked = asked_of(a, row);
  const float* const most = a.most + row * a.splits;
  float m = -INFINITY;
  for (int i = 0; i < a.splits; ++i) m = fmaxf(m, most[i]);
  uint32_t count = 0;
  u64 mass = 0;
  const int64_t mine = row * a.splits * kBins + kBins - 1 - (int)threadIdx.x;
  for (int i = 0; i < a.splits; ++i) {
    count += a.count[mine + (int64_t)i * kBins];
    const u64 w = a.mass[mine + (int64_t)i * kBins];
    // Each part's sums are relative to its own largest logit.
    mass += most[i] == m || w == 0 ? w : __double2ull_rn((double)w * weight(most[i], m, asked.c));
  }
  select<T>(a, row, m, asked, count, mass, s);
}

// Parts of a row: a workgroup for each compute unit, within bounds: a histogram
// costs its second launch 0.3 us, and one of fewer logits is hardly shorter (one row
// of 32000 fp16 in 2, 4 and 8 parts 19.1, 17.9 and 18.6 us, of 131072 in 8, 16 and 32
// 25.4, 26.1 and 30.6).
int choose_splits(const SampleTokens& c) {
  const int64_t want = device_cus() / c.M, most = ((int64_t)c.V + kMinPart - 1) / kMinPart;
  const int64_t parts = most < kMaxParts ? most : kMaxParts;
  return (int)(want < 1 ? 1 : want < parts ? want : parts);
}

template <typename T>
hipError_t launch(const SampleArgs& a, hipStream_t stream) {
  if (a.splits == 1) {
    // A launch holds less than 2^32 threads.
    constexpr int64_t kMostRows = 0xFFFFFFFFll / kThreads;
    for (int64_t first = 0; first < a.M; first += kMostRows) {
      const int64_t rows = a.M - first < kMostRows ? a.M - first : kMostRows;
      sample_kernel<T><<<(unsigned)rows, kThreads, 0, stream>>>(a, first);
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
    return hipSuccess;
  }
  const unsigned grid = (unsigned)((a.M + kXcds - 1) / kXcds * kXcds * a.splits);
  sample_histogram_kernel<T><<<grid, kThreads, 0, stream>>>(a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  sample_select_kernel<T><<<(unsigned)a.M, kThreads, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace

int64_t sample_tokens_workspace(const SampleTokens& c) {
  const int64_t splits = choose_splits(c);
  return splits == 1 ? 0 : c.M * splits * (kBins * 12 + 4);
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
  a.one = 1ull << e;
  a.unit = (double)a.one;
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
