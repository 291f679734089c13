// Log probabilities of given tokens, the entropy of each row's distribution
// and its most likely alternatives, from logits x [M, V]:
//
//   m = max x,  l = sum exp(x - m),  lse = m + log l
//   logprob  = x_token - lse
//   entropy  = log l - sum exp(x - m) (x - m) / l
//   top      = the `top` largest x (ties: the lowest index first), minus lse
//
// Sums in fp32, with their running maximum.  Logits of -inf are masked: they
// weigh nothing and have log probability -inf; a row of them alone has entropy
// 0 and log probabilities -inf.
//
// One read of the logits.  A workgroup walks a part of a row in chunks of 8192
// logits in registers, from which it takes the sums and, against the running
// list of the best `top`, the few logits that enter it.  Rows are split over
// workgroups while there are too few of them; a second launch then joins the
// parts.  Without alternatives 256 threads hold 32 logits each: 2047 x 100003
// fp32 take 143 us, 5.7 of a plain read's 7.1 TB/s, bound by bytes.  With them 512 hold 16, so that
// the work that a row needs once (bound, ranks, join) is spread wider: 64 x
// 131072 fp16 with 20 alternatives take 22.3 us, bound by the latency of those
// chains in two launches (27 us with 256 threads, 27.6 with 1024).
#include "internal.h"
#include "wave_device.h"

namespace dptq {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kChunk = 8192;
constexpr int kTopThreads = 512, kSumThreads = 256;
constexpr int kTopPer = kChunk / kTopThreads;   // logits of a thread in a chunk
constexpr int kGroups = 256;                    // whose maxima bound the list
constexpr int kCap = 512;                       // candidates of a chunk that are ranked at once
constexpr int kMaxTop = 64;

struct LogprobArgs {
  const void* x;
  int64_t ld, M;
  int V, top, splits;
  const int64_t* tokens;
  float *logprobs, *entropy, *top_logprobs;
  int64_t* top_ids;
  float4* part;   // [M][splits] (m, l, u, -)
  unsigned long long* list;   // [M][splits][top] keys
};

// Sums relative to the maximum m: l = sum exp(x - m), u = sum exp(x - m) (x - m).
struct Stats {
  float m, l, u;
};

__device__ __forceinline__ Stats join(Stats a, Stats b) {
  const float m = fmaxf(a.m, b.m);
  const float ra = a.m == m ? 0.0f : a.m - m, rb = b.m == m ? 0.0f : b.m - m;   // 0 also for -inf - -inf
  const float fa = __builtin_amdgcn_exp2f(ra * kLog2e), fb = __builtin_amdgcn_exp2f(rb * kLog2e);
  // Where a factor is 0 its difference may be infinite.
  const float ua = fa > 0.0f ? fa * (a.u + a.l * ra) : 0.0f, ub = fb > 0.0f ? fb * (b.u + b.l * rb) : 0.0f;
  return Stats{m, fa * a.l + fb * b.l, ua + ub};
}

// The sums of a thread's values; -inf weighs nothing, NaN makes them NaN.
template <int PER>
__device__ __forceinline__ Stats stats_of(const float (&v)[PER]) {
  float m = v[0];
#pragma unroll
  for (int i = 1; i < PER; ++i) m = fmaxf(m, v[i]);
  const float base = m == -INFINITY ? 0.0f : m;
  float l[2] = {0.0f, 0.0f}, u[2] = {0.0f, 0.0f};
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const float d = v[i] - base;
    const float e = __builtin_amdgcn_exp2f(d * kLog2e);
    l[i & 1] += e;
    u[i & 1] = fmaf(e, fmaxf(d, -200.0f), u[i & 1]);   // e is 0 below that: no 0 * -inf
  }
  return Stats{m, l[0] + l[1], u[0] + u[1]};
}

// Over a workgroup of WAVES waves; every thread has the result.  The maximum
// first, then the sums relative to it.
template <int WAVES>
__device__ __forceinline__ Stats block_join(Stats s, Stats* part) {
  const auto wave_join = [](Stats s) {
    s = join(s, Stats{wave_max(s.m), 0.0f, 0.0f});
    return Stats{s.m, wave_sum(s.l), wave_sum(s.u)};
  };
  s = wave_join(s);
  if (WAVES == 1) return s;
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = s;
  __syncthreads();
  return wave_join((int)(threadIdx.x & 63) < WAVES ? part[threadIdx.x & 63] : Stats{-INFINITY, 0.0f, 0.0f});
}

// A logit and its index as one number: larger ones come first, equal logits by
// index.  0: none.
using Key = unsigned long long;

__device__ __forceinline__ uint32_t ordered(float x) {
  const uint32_t u = __float_as_uint(x + 0.0f);   // -0 is 0
  return u ^ (u >> 31 ? 0xFFFFFFFFu : 0x80000000u);
}
__device__ __forceinline__ float unordered(uint32_t o) { return __uint_as_float(o ^ (o >> 31 ? 0x80000000u : 0xFFFFFFFFu)); }
__device__ __forceinline__ Key key_of(float x, int i) { return (Key)ordered(x) << 32 | (uint32_t)~i; }
__device__ __forceinline__ float key_value(Key k) { return k ? unordered((uint32_t)(k >> 32)) : -INFINITY; }
__device__ __forceinline__ int key_index(Key k) { return k ? (int)~(uint32_t)k : 0x7FFFFFFF; }

constexpr uint32_t kOrderedLowest = 0x007FFFFFu;   // of -inf

struct TopScratch {
  Key best[kMaxTop];   // the list so far, in order, 0 where it has room
  Key next[kMaxTop];
  Key found[kCap + kMaxTop];
  uint32_t group[kGroups];
  Key wave_best[kTopThreads / 64];
  uint32_t bound;
  int count;
};

__device__ __forceinline__ void clear_list(TopScratch& t, int top) {
  if ((int)threadIdx.x < top) t.best[threadIdx.x] = 0;
  if (threadIdx.x == 0) t.count = 0;
  __syncthreads();
}

// Merges a chunk into the list: index(k) is that of the thread's value v[k],
// negative where it has none (whole: it has all); mine_top the largest of them,
// of what has no index also.  Indices of later chunks are larger, so a value
// enters only if it is larger than the list's last, or if the list has room.
//
// Where too many would (the first chunk of a row), the `top`-th largest of the
// maxima of 256 groups of threads, to 16 bits, is a bound that at least
// `top` values reach, and few more do in ordinary data.  Where that is too many
// as well (ties), the entries are taken out one by one.
template <typename Index>
__device__ __forceinline__ void merge_chunk(const float (&v)[kTopPer], float mine_top, const Index& index,
                                            bool whole, int top, TopScratch& t) {
  const Key last = t.best[top - 1];
  const bool room = last == 0;
  // Larger than the last: at least the next float.
  const float least = room ? -INFINITY : unordered((uint32_t)(last >> 32) + 1);
  uint32_t mine = 0;
  const auto choose = [&](float bound) {
    mine = 0;
    if (!__any(mine_top >= bound)) return;   // most waves, in most chunks
#pragma unroll
    for (int k = 0; k < kTopPer; ++k) mine |= v[k] >= bound && (whole || index(k) >= 0) ? 1u << k : 0u;
  };
  const auto gather = [&]() {
    if (mine) {
      int at = atomicAdd(&t.count, __popc(mine));
#pragma unroll
      for (int k = 0; k < kTopPer; ++k)
        if (mine >> k & 1) {
          if (at < kCap) t.found[at] = key_of(v[k], index(k));
          ++at;
        }
    }
    __syncthreads();
    return t.count;
  };
  int n = 0;
  if (!room) {
    choose(least);
    n = gather();
  }
  if (room || n > kCap) {   // the same for every thread
    // In a chunk with places that have no index only the others count.
    uint32_t high = 0;
    if (whole) {
      high = mine_top >= least ? ordered(mine_top) : 0;
    } else {
#pragma unroll
      for (int k = 0; k < kTopPer; ++k)
        if (v[k] >= least && index(k) >= 0) high = max(high, ordered(v[k]));
    }
    constexpr int kMates = kTopThreads / kGroups;
#pragma unroll
    for (int off = 1; off < kMates; off *= 2) high = max(high, (uint32_t)__shfl_xor((int)high, off));
    if (threadIdx.x % kMates == 0) t.group[threadIdx.x / kMates] = high;
    __syncthreads();
    if (threadIdx.x < 64) {
      const uint4 g = *reinterpret_cast<const uint4*>(t.group + 4 * threadIdx.x);
      uint32_t bound = 0;
      for (int bit = 31; bit >= 16; --bit) {
        const uint32_t b = bound | 1u << bit;
        const int reach = __popcll(__ballot(g.x >= b)) + __popcll(__ballot(g.y >= b)) +
                          __popcll(__ballot(g.z >= b)) + __popcll(__ballot(g.w >= b));
        if (reach >= top) bound = b;
      }
      if (threadIdx.x == 0) {
        t.bound = bound > kOrderedLowest ? bound : kOrderedLowest;
        t.count = 0;
      }
    }
    __syncthreads();
    choose(fmaxf(least, unordered(t.bound)));
    n = gather();
  }
  if (n == 0) {   // and so is count
    __syncthreads();
    return;
  }
  if (n <= kCap) {
    // Ranks of the candidates and of the list's entries among all of them: 16
    // threads count for one.
    if ((int)threadIdx.x < top) {
      t.found[n + threadIdx.x] = t.best[threadIdx.x];
      t.next[threadIdx.x] = 0;
    }
    __syncthreads();
    const int all = n + top;
    for (int c = threadIdx.x / 16; c < all; c += kTopThreads / 16) {
      const Key mine_key = t.found[c];
      int rank = 0;
      for (int o = threadIdx.x % 16; o < all; o += 16) rank += t.found[o] > mine_key;
#pragma unroll
      for (int off = 8; off > 0; off >>= 1) rank += __shfl_xor(rank, off);
      if (threadIdx.x % 16 == 0 && mine_key && rank < top) t.next[rank] = mine_key;
    }
    __syncthreads();
  } else {
    // One by one: the best of the chunk after the last one taken, against the
    // head of the list.
    Key taken = ~(Key)0;
    int head = 0;
    for (int out = 0; out < top; ++out) {
      Key best = 0;
#pragma unroll
      for (int k = 0; k < kTopPer; ++k)
        if (mine >> k & 1) {
          const Key c = key_of(v[k], index(k));
          if (c < taken && c > best) best = c;
        }
#pragma unroll
      for (int off = 32; off > 0; off >>= 1) {
        const Key other = __shfl_xor(best, off);
        if (other > best) best = other;
      }
      if ((threadIdx.x & 63) == 0) t.wave_best[threadIdx.x >> 6] = best;
      __syncthreads();
      for (int w = 0; w < kTopThreads / 64; ++w)
        if (t.wave_best[w] > best) best = t.wave_best[w];
      const Key old = t.best[head];
      if (threadIdx.x == 0) t.next[out] = old > best ? old : best;
      if (old > best) ++head;
      else taken = best;
      __syncthreads();
    }
  }
  if ((int)threadIdx.x < top) t.best[threadIdx.x] = t.next[threadIdx.x];
  if (threadIdx.x == 0) t.count = 0;
  __syncthreads();
}

__device__ __forceinline__ float value(const __half* p) { return __half2float(*p); }
__device__ __forceinline__ float value(const float* p) { return *p; }

__device__ __forceinline__ void unpack(const uint4 r, const __half*, float* v) {
  const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    v[2 * j] = __half2float(__ushort_as_half((unsigned short)(w[j] & 0xFFFFu)));
    v[2 * j + 1] = __half2float(__ushort_as_half((unsigned short)(w[j] >> 16)));
  }
}
__device__ __forceinline__ void unpack(const uint4 r, const float*, float* v) {
  v[0] = __uint_as_float(r.x);
  v[1] = __uint_as_float(r.y);
  v[2] = __uint_as_float(r.z);
  v[3] = __uint_as_float(r.w);
}

// The row's token and its logit, for thread 0; fetched ahead of the row.
struct Picked {
  int64_t token;
  float x;
};
template <typename T>
__device__ __forceinline__ Picked pick(const LogprobArgs& a, int64_t row) {
  Picked p{-1, 0.0f};
  if (threadIdx.x == 0) {
    p.token = a.tokens[row];
    if (p.token >= 0 && p.token < a.V) p.x = value(static_cast<const T*>(a.x) + row * a.ld + p.token);
  }
  return p;
}

// The row's results from its sums and list (thread 0, and a thread an entry).
__device__ __forceinline__ void finish(const LogprobArgs& a, int64_t row, Picked p, Stats s, const Key* best) {
  const float log_l = logf(s.l);
  if (threadIdx.x == 0) {
    float lp = 0.0f;
    if (p.token >= a.V) lp = NAN;
    else if (p.token >= 0) lp = p.x == -INFINITY ? p.x : (p.x - s.m) - log_l;
    a.logprobs[row] = lp;
    a.entropy[row] = s.l == 0.0f ? 0.0f : log_l - s.u / s.l;   // 0: all masked
  }
  if ((int)threadIdx.x < a.top) {
    const float x = key_value(best[threadIdx.x]);
    a.top_logprobs[row * a.top + threadIdx.x] = x == -INFINITY ? x : (x - s.m) - log_l;
    a.top_ids[row * a.top + threadIdx.x] = min(key_index(best[threadIdx.x]), a.V - 1);   // NaN takes no place
  }
}

// Grid: (splits, rows at a time).  The row as 16-byte units from the aligned address at or
// before its first element: units that reach over an end are loaded element by
// element.
template <typename T, bool TOP>
__global__ void __launch_bounds__(TOP ? kTopThreads : kSumThreads, TOP ? kTopThreads / 128 : 8) token_logprobs_kernel(LogprobArgs a) {
  constexpr int kThreads = TOP ? kTopThreads : kSumThreads, kPer = kChunk / kThreads;
  constexpr int E = 16 / sizeof(T), kUnits = kPer / E;
  __shared__ Stats part[kThreads / 64];
  __shared__ TopScratch scratch;
  for (int64_t row = blockIdx.y; row < a.M; row += gridDim.y) {
    const T* const x = static_cast<const T*>(a.x) + row * a.ld;
    const int skew = (int)(reinterpret_cast<uintptr_t>(x) & 15u) / (int)sizeof(T);
    const int chunks = (int)(((int64_t)a.V + skew + kChunk - 1) / kChunk);
    const int begin = (int)((int64_t)chunks * blockIdx.x / a.splits);
    const int end = (int)((int64_t)chunks * (blockIdx.x + 1) / a.splits);
    const Picked picked = a.splits == 1 ? pick<T>(a, row) : Picked{-1, 0.0f};
    Stats s{-INFINITY, 0.0f, 0.0f};
    if constexpr (TOP) clear_list(scratch, a.top);
    for (int c = begin; c < end; ++c) {
      float v[kPer];
      const int first = c * kChunk - skew;   // of the chunk; may be negative
      const int mine = first + (int)threadIdx.x * E;
#pragma unroll
      for (int n = 0; n < kUnits; ++n) {
        const int i = mine + n * kThreads * E;
        if (i >= 0 && i + E <= a.V) {
          unpack(*reinterpret_cast<const uint4*>(x + i), x, v + n * E);
        } else {
#pragma unroll
          for (int j = 0; j < E; ++j) v[n * E + j] = i + j >= 0 && i + j < a.V ? value(x + i + j) : -INFINITY;
        }
      }
      const Stats here = stats_of(v);
      s = join(s, here);
      if constexpr (TOP) {
        const auto index = [&](int k) {
          const int i = mine + (k / E) * kThreads * E + k % E;
          return i < a.V ? i : -1;
        };
        merge_chunk(v, here.m, index, first >= 0 && first + kChunk <= a.V, a.top, scratch);
      }
    }
    s = block_join<kThreads / 64>(s, part);
    if (a.splits == 1) {
      finish(a, row, picked, s, TOP ? scratch.best : nullptr);
    } else {
      const int64_t at = row * a.splits + blockIdx.x;
      if (threadIdx.x == 0) a.part[at] = make_float4(s.m, s.l, s.u, 0.0f);
      if (TOP && (int)threadIdx.x < a.top) a.list[at * a.top + threadIdx.x] = scratch.best[threadIdx.x];
    }
    __syncthreads();   // part and the list are free again
  }
}

// Joins a row's parts, which lie in the order of their indices.
template <typename T, bool TOP>
__global__ void __launch_bounds__(TOP ? kTopThreads : 64) join_logprobs_kernel(LogprobArgs a) {
  constexpr int kThreads = TOP ? kTopThreads : 64;
  __shared__ Stats part[kThreads / 64];
  __shared__ TopScratch scratch;
  for (int64_t row = blockIdx.x; row < a.M; row += gridDim.x) {
    const Picked picked = pick<T>(a, row);
    Stats s{-INFINITY, 0.0f, 0.0f};
    for (int i = threadIdx.x; i < a.splits; i += kThreads) {
      const float4 p = a.part[row * a.splits + i];
      s = join(s, Stats{p.x, p.y, p.z});
    }
    s = block_join<kThreads / 64>(s, part);
    if constexpr (TOP) {
      clear_list(scratch, a.top);
      const int n = a.splits * a.top;
      const Key* const list = a.list + row * n;
      for (int c = 0; c < n; c += kChunk) {
        float v[kTopPer];
        int id[kTopPer];
#pragma unroll
        for (int k = 0; k < kTopPer; ++k) {
          const int i = c + k * kThreads + (int)threadIdx.x;
          const Key e = i < n ? list[i] : 0;
          id[k] = e ? key_index(e) : -1;
          v[k] = key_value(e);
        }
        float most = v[0];
#pragma unroll
        for (int k = 1; k < kTopPer; ++k) most = fmaxf(most, v[k]);
        merge_chunk(v, most, [&](int k) { return id[k]; }, false, a.top, scratch);
      }
    }
    finish(a, row, picked, s, TOP ? scratch.best : nullptr);
    __syncthreads();
  }
}

// Parts of a row: enough workgroups for 8 of 256 threads, or with alternatives
// the two of 512 that it holds, on each compute unit, of one chunk or more.
int choose_splits(const TokenLogprobs& c) {
  const int64_t chunks = ((int64_t)c.V + kChunk - 1) / kChunk;
  const int64_t want = ((c.top ? 2 : 8) * (int64_t)device_cus() + c.M - 1) / c.M;
  return (int)(want < chunks ? want : chunks);
}

template <typename T, bool TOP>
hipError_t launch(const LogprobArgs& a, hipStream_t stream) {
  const unsigned rows = (unsigned)(a.M < 65535 ? a.M : 65535);
  constexpr int kThreads = TOP ? kTopThreads : kSumThreads, kJoinThreads = TOP ? kTopThreads : 64;
  token_logprobs_kernel<T, TOP><<<dim3((unsigned)a.splits, rows), kThreads, 0, stream>>>(a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.splits == 1) return e;
  join_logprobs_kernel<T, TOP><<<rows, kJoinThreads, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace

int64_t token_logprobs_workspace(const TokenLogprobs& c) {
  const int64_t splits = choose_splits(c);
  return splits == 1 ? 0 : c.M * splits * (16 + 8 * (int64_t)c.top);
}

hipError_t launch_token_logprobs(const TokenLogprobs& c, hipStream_t stream) {
  LogprobArgs a{c.logits, c.ld, c.M, c.V, c.top, choose_splits(c), c.tokens, c.logprobs, c.entropy,
                c.top_logprobs, c.top_ids, nullptr, nullptr};
  a.part = static_cast<float4*>(c.workspace);
  a.list = reinterpret_cast<Key*>(a.part + a.M * a.splits);
  if (c.fp32) return c.top ? launch<float, true>(a, stream) : launch<float, false>(a, stream);
  return c.top ? launch<__half, true>(a, stream) : launch<__half, false>(a, stream);
}

}  // namespace dptq
