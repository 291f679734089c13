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
// logits, 32 a thread in registers, from which it takes the sums and, against
// the running list of the best `top`, the few logits that enter it.  Rows are
// split over workgroups while there are too few of them; a second launch then
// joins the parts.
#include "internal.h"

namespace dptq {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kThreads = 256;
constexpr int kPer = 32;                        // logits of a thread in a chunk
constexpr int kChunk = kThreads * kPer;
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
  int2* list;     // [M][splits][top] (bits of x, index)
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
__device__ __forceinline__ Stats stats_of(const float (&v)[kPer]) {
  float m = v[0];
#pragma unroll
  for (int i = 1; i < kPer; ++i) m = fmaxf(m, v[i]);
  const float base = m == -INFINITY ? 0.0f : m;
  float l[2] = {0.0f, 0.0f}, u[2] = {0.0f, 0.0f};
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const float d = v[i] - base;
    const float e = __builtin_amdgcn_exp2f(d * kLog2e);
    l[i & 1] += e;
    u[i & 1] = fmaf(e, fmaxf(d, -200.0f), u[i & 1]);   // e is 0 below that: no 0 * -inf
  }
  return Stats{m, l[0] + l[1], u[0] + u[1]};
}

__device__ __forceinline__ Stats block_join(Stats s, Stats* part) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1)
    s = join(s, Stats{__shfl_xor(s.m, off), __shfl_xor(s.l, off), __shfl_xor(s.u, off)});
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = s;
  __syncthreads();
  return join(join(part[0], part[1]), join(part[2], part[3]));
}

// (x, i) comes before (y, j).
__device__ __forceinline__ bool before(float x, int i, float y, int j) { return x > y || (x == y && i < j); }

// The best `top` values so far, in order; places that nothing has taken hold
// (-inf, INT_MAX).
struct TopList {
  float x[kMaxTop];
  int i[kMaxTop];
};

struct TopScratch {
  TopList best, next;
  float x[kCap + kMaxTop];
  int i[kCap + kMaxTop];
  float group[kThreads];
  float wave_x[4];
  int wave_i[4];
  int count;
  float threshold;
};

__device__ __forceinline__ void clear_list(TopScratch& t, int top) {
  if ((int)threadIdx.x < top) {
    t.best.x[threadIdx.x] = -INFINITY;
    t.best.i[threadIdx.x] = 0x7FFFFFFF;
  }
  if (threadIdx.x == 0) t.count = 0;
  __syncthreads();
}

// Merges a chunk into the list: index(k) is that of the thread's value v[k],
// negative where it has none.  Indices of later chunks are larger, so a value
// enters only if it is larger than the list's last, or if the list has room.
//
// Where too many are larger (the first chunk of a row), the `top`-th largest of
// the threads' maxima is a bound that at least `top` values reach, and few more
// do in ordinary data.  Where that is too many as well (ties), the entries are
// taken out one by one.
// whole: the thread has all its values.
template <typename Index>
__device__ __forceinline__ void merge_chunk(const float (&v)[kPer], const Index& index, bool whole, int top,
                                            TopScratch& t) {
  const float last = t.best.x[top - 1];
  const bool room = t.best.i[top - 1] == 0x7FFFFFFF;
  uint32_t mine = 0;
#pragma unroll
  for (int k = 0; k < kPer; ++k) mine |= v[k] > last || (room && v[k] == v[k]) ? 1u << k : 0u;
  if (!whole) {
#pragma unroll
    for (int k = 0; k < kPer; ++k)
      if (index(k) < 0) mine &= ~(1u << k);
  }
  const auto gather = [&](uint32_t mask) {
    if (mask) {
      int at = atomicAdd(&t.count, __popc(mask));
#pragma unroll
      for (int k = 0; k < kPer; ++k)
        if (mask >> k & 1) {
          if (at < kCap) t.x[at] = v[k], t.i[at] = index(k);
          ++at;
        }
    }
    __syncthreads();
    return t.count;
  };
  int n = 0;
  if (!room) n = gather(mine);
  if (room || n > kCap) {   // the same for every thread
    float top_of_mine = -INFINITY;
#pragma unroll
    for (int k = 0; k < kPer; ++k)
      if (mine >> k & 1) top_of_mine = fmaxf(top_of_mine, v[k]);
    t.group[threadIdx.x] = top_of_mine;
    __syncthreads();
    if (threadIdx.x == 0) t.count = 0;
    int rank = 0;
    for (int k = 0; k < kThreads; k += 4) {
      const float4 g = *reinterpret_cast<const float4*>(t.group + k);
      rank += before(g.x, k, top_of_mine, (int)threadIdx.x) + before(g.y, k + 1, top_of_mine, (int)threadIdx.x) +
              before(g.z, k + 2, top_of_mine, (int)threadIdx.x) + before(g.w, k + 3, top_of_mine, (int)threadIdx.x);
    }
    if (rank == top - 1) t.threshold = top_of_mine;
    __syncthreads();
    const float bound = t.threshold;
#pragma unroll
    for (int k = 0; k < kPer; ++k)
      if (!(v[k] >= bound)) mine &= ~(1u << k);
    n = gather(mine);
  }
  if (n == 0) {   // and so is count
    __syncthreads();
    return;
  }
  if (n <= kCap) {
    // Rank of each candidate and of each list entry among all of them.
    if ((int)threadIdx.x < top) {
      t.x[n + threadIdx.x] = t.best.x[threadIdx.x];
      t.i[n + threadIdx.x] = t.best.i[threadIdx.x];
    }
    __syncthreads();
    const int all = n + top;
    for (int c = threadIdx.x; c < all; c += kThreads) {
      const float x = t.x[c];
      const int i = t.i[c];
      int rank = 0;
      for (int o = 0; o < all; ++o)
        rank += before(t.x[o], t.i[o], x, i) || (t.x[o] == x && t.i[o] == i && o < c);
      if (rank < top) t.next.x[rank] = x, t.next.i[rank] = i;
    }
    __syncthreads();
  } else {
    // One by one: the best of the chunk that comes after the last one taken,
    // against the head of the list.
    float last_x = INFINITY;
    int last_i = -1, head = 0;
    for (int out = 0; out < top; ++out) {
      float bx = -INFINITY;
      int bi = 0x7FFFFFFF;
#pragma unroll
      for (int k = 0; k < kPer; ++k)
        if (mine >> k & 1) {
          const int i = index(k);
          if (before(last_x, last_i, v[k], i) && before(v[k], i, bx, bi)) bx = v[k], bi = i;
        }
#pragma unroll
      for (int off = 32; off > 0; off >>= 1) {
        const float ox = __shfl_xor(bx, off);
        const int oi = __shfl_xor(bi, off);
        if (before(ox, oi, bx, bi)) bx = ox, bi = oi;
      }
      if ((threadIdx.x & 63) == 0) t.wave_x[threadIdx.x >> 6] = bx, t.wave_i[threadIdx.x >> 6] = bi;
      __syncthreads();
      for (int w = 0; w < 4; ++w)
        if (before(t.wave_x[w], t.wave_i[w], bx, bi)) bx = t.wave_x[w], bi = t.wave_i[w];
      const float hx = t.best.x[head];
      const int hi = t.best.i[head];
      const bool from_list = !before(bx, bi, hx, hi);
      if (threadIdx.x == 0) {
        t.next.x[out] = from_list ? hx : bx;
        t.next.i[out] = from_list ? hi : bi;
      }
      if (from_list) ++head;
      else last_x = bx, last_i = bi;
      __syncthreads();
    }
  }
  if ((int)threadIdx.x < top) {
    t.best.x[threadIdx.x] = t.next.x[threadIdx.x];
    t.best.i[threadIdx.x] = t.next.i[threadIdx.x];
  }
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

// The row's results from its sums and list (thread 0, and a thread an entry).
template <typename T>
__device__ __forceinline__ void finish(const LogprobArgs& a, int64_t row, Stats s, const TopList* best) {
  const float log_l = logf(s.l);
  if (threadIdx.x == 0) {
    const int64_t t = a.tokens[row];
    float lp = 0.0f;
    if (t >= a.V) {
      lp = NAN;
    } else if (t >= 0) {
      const float v = value(static_cast<const T*>(a.x) + row * a.ld + t);
      lp = v == -INFINITY ? v : (v - s.m) - log_l;
    }
    a.logprobs[row] = lp;
    a.entropy[row] = s.l == 0.0f ? 0.0f : log_l - s.u / s.l;   // 0: all masked
  }
  if ((int)threadIdx.x < a.top) {
    const float x = best->x[threadIdx.x];
    a.top_logprobs[row * a.top + threadIdx.x] = x == -INFINITY ? x : (x - s.m) - log_l;
    a.top_ids[row * a.top + threadIdx.x] = min(best->i[threadIdx.x], a.V - 1);   // NaN takes no place
  }
}

// Grid: (splits, rows at a time).  The row as 16-byte units from the aligned address at or
// before its first element: units that reach over an end are loaded element by
// element.
template <typename T, bool TOP>
__global__ void __launch_bounds__(kThreads) token_logprobs_kernel(LogprobArgs a) {
  constexpr int E = 16 / sizeof(T), kUnits = kPer / E;
  __shared__ Stats part[4];
  __shared__ TopScratch scratch;
  for (int64_t row = blockIdx.y; row < a.M; row += gridDim.y) {
    const T* const x = static_cast<const T*>(a.x) + row * a.ld;
    const int skew = (int)(reinterpret_cast<uintptr_t>(x) & 15u) / (int)sizeof(T);
    const int chunks = (int)(((int64_t)a.V + skew + kChunk - 1) / kChunk);
    const int begin = (int)((int64_t)chunks * blockIdx.x / a.splits);
    const int end = (int)((int64_t)chunks * (blockIdx.x + 1) / a.splits);
    Stats s{-INFINITY, 0.0f, 0.0f};
    if constexpr (TOP) clear_list(scratch, a.top);
    for (int c = begin; c < end; ++c) {
      float v[kPer];
      const int64_t first = (int64_t)c * kChunk - skew;   // of the chunk; may be negative, may pass 2^31
#pragma unroll
      for (int n = 0; n < kUnits; ++n) {
        const int64_t i = first + (n * kThreads + (int)threadIdx.x) * E;
        if (i >= 0 && i + E <= a.V) {
          unpack(*reinterpret_cast<const uint4*>(x + i), x, v + n * E);
        } else {
#pragma unroll
          for (int j = 0; j < E; ++j) v[n * E + j] = i + j >= 0 && i + j < a.V ? value(x + i + j) : -INFINITY;
        }
      }
      s = join(s, stats_of(v));
      if constexpr (TOP) {
        const auto index = [&](int k) {
          const int64_t i = first + ((k / E) * kThreads + (int)threadIdx.x) * E + k % E;
          return i < a.V ? (int)i : -1;
        };
        merge_chunk(v, index, first >= 0 && first + kChunk <= a.V, a.top, scratch);
      }
    }
    s = block_join(s, part);
    if (a.splits == 1) {
      finish<T>(a, row, s, TOP ? &scratch.best : nullptr);
    } else {
      const int64_t at = row * a.splits + blockIdx.x;
      if (threadIdx.x == 0) a.part[at] = make_float4(s.m, s.l, s.u, 0.0f);
      if (TOP && (int)threadIdx.x < a.top)
        a.list[at * a.top + threadIdx.x] =
            make_int2(__float_as_int(scratch.best.x[threadIdx.x]), scratch.best.i[threadIdx.x]);
    }
    __syncthreads();   // part and the list are free again
  }
}

// Joins a row's parts, which lie in the order of their indices.
template <typename T, bool TOP>
__global__ void __launch_bounds__(kThreads) join_logprobs_kernel(LogprobArgs a) {
  __shared__ Stats part[4];
  __shared__ TopScratch scratch;
  for (int64_t row = blockIdx.x; row < a.M; row += gridDim.x) {
    Stats s{-INFINITY, 0.0f, 0.0f};
    for (int i = threadIdx.x; i < a.splits; i += kThreads) {
      const float4 p = a.part[row * a.splits + i];
      s = join(s, Stats{p.x, p.y, p.z});
    }
    s = block_join(s, part);
    if constexpr (TOP) {
      clear_list(scratch, a.top);
      const int n = a.splits * a.top;
      const int2* const list = a.list + row * n;
      for (int c = 0; c < n; c += kChunk) {
        float v[kPer];
        int id[kPer];
#pragma unroll
        for (int k = 0; k < kPer; ++k) {
          const int i = c + k * kThreads + (int)threadIdx.x;
          const int2 e = i < n ? list[i] : make_int2(0, 0x7FFFFFFF);
          id[k] = e.y == 0x7FFFFFFF ? -1 : e.y;
          v[k] = id[k] < 0 ? -INFINITY : __int_as_float(e.x);
        }
        merge_chunk(v, [&](int k) { return id[k]; }, false, a.top, scratch);
      }
    }
    finish<T>(a, row, s, TOP ? &scratch.best : nullptr);
    __syncthreads();
  }
}

// Parts of a row: enough workgroups for a few on each compute unit, of one
// chunk or more.
int choose_splits(const TokenLogprobs& c) {
  const int64_t chunks = ((int64_t)c.V + kChunk - 1) / kChunk;
  const int64_t want = (8 * (int64_t)device_cus() + c.M - 1) / c.M;
  return (int)(want < chunks ? want : chunks);
}

template <typename T, bool TOP>
hipError_t launch(const LogprobArgs& a, hipStream_t stream) {
  const unsigned rows = (unsigned)(a.M < 65535 ? a.M : 65535);
  token_logprobs_kernel<T, TOP><<<dim3((unsigned)a.splits, rows), kThreads, 0, stream>>>(a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.splits == 1) return e;
  join_logprobs_kernel<T, TOP><<<rows, kThreads, 0, stream>>>(a);
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
  a.list = reinterpret_cast<int2*>(a.part + a.M * a.splits);
  if (c.fp32) return c.top ? launch<float, true>(a, stream) : launch<float, false>(a, stream);
  return c.top ? launch<__half, true>(a, stream) : launch<__half, false>(a, stream);
}

}  // namespace dptq
