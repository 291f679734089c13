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
#include "internal.h"

namespace dptq {
namespace {

constexpr float kLog2e = 1.4426950408889634f;

struct LogprobArgs {
  const void* x;
  int64_t ld, M;
  int V, top;
  const int64_t* tokens;
  float *logprobs, *entropy, *top_logprobs;
  int64_t* top_ids;
};

__device__ __forceinline__ float value(const __half* p) { return __half2float(*p); }
__device__ __forceinline__ float value(const float* p) { return *p; }

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

// (x, i) comes before (y, j).
__device__ __forceinline__ bool before(float x, int i, float y, int j) { return x > y || (x == y && i < j); }

template <typename T>
__global__ void __launch_bounds__(256) token_logprobs_kernel(LogprobArgs a) {
  __shared__ Stats part[4];
  __shared__ float best_x[4];
  __shared__ int best_i[4];
  const int64_t row = blockIdx.x;
  const T* const x = static_cast<const T*>(a.x) + row * a.ld;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  Stats s{-INFINITY, 0.0f, 0.0f};
  for (int i = threadIdx.x; i < a.V; i += 256) {
    const float v = value(x + i);
    if (v != -INFINITY) s = join(s, Stats{v, 1.0f, 0.0f});
  }
#pragma unroll
  for (int off = 32; off > 0; off >>= 1)
    s = join(s, Stats{__shfl_xor(s.m, off), __shfl_xor(s.l, off), __shfl_xor(s.u, off)});
  if (lane == 0) part[wave] = s;
  __syncthreads();
  s = join(join(part[0], part[1]), join(part[2], part[3]));
  const float log_l = logf(s.l), max_x = s.m;
  if (threadIdx.x == 0) {
    const int64_t t = a.tokens[row];
    float lp = 0.0f;
    if (t >= a.V) lp = NAN;
    else if (t >= 0) {
      const float v = value(x + t);
      lp = v == -INFINITY ? v : (v - max_x) - log_l;
    }
    a.logprobs[row] = lp;
    a.entropy[row] = s.m == -INFINITY ? 0.0f : log_l - s.u / s.l;
  }
  float last_x = INFINITY;
  int last_i = -1;
  for (int k = 0; k < a.top; ++k) {
    float bx = -INFINITY;
    int bi = a.V;
    for (int i = threadIdx.x; i < a.V; i += 256) {
      const float v = value(x + i);
      if (before(last_x, last_i, v, i) && before(v, i, bx, bi)) bx = v, bi = i;
    }
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) {
      const float ox = __shfl_xor(bx, off);
      const int oi = __shfl_xor(bi, off);
      if (before(ox, oi, bx, bi)) bx = ox, bi = oi;
    }
    if (lane == 0) best_x[wave] = bx, best_i[wave] = bi;
    __syncthreads();
    for (int w = 0; w < 4; ++w)
      if (before(best_x[w], best_i[w], bx, bi)) bx = best_x[w], bi = best_i[w];
    __syncthreads();
    last_x = bx, last_i = bi;
    if (threadIdx.x == 0) {
      a.top_logprobs[row * a.top + k] = bx == -INFINITY ? bx : (bx - max_x) - log_l;
      a.top_ids[row * a.top + k] = min(bi, a.V - 1);   // NaN is never taken
    }
  }
}

}  // namespace

int64_t token_logprobs_workspace(const TokenLogprobs&) { return 0; }

hipError_t launch_token_logprobs(const TokenLogprobs& c, hipStream_t stream) {
  LogprobArgs a{c.logits, c.ld, c.M, c.V, c.top, c.tokens, c.logprobs, c.entropy, c.top_logprobs, c.top_ids};
  if (c.fp32)
    token_logprobs_kernel<float><<<(unsigned)c.M, 256, 0, stream>>>(a);
  else
    token_logprobs_kernel<__half><<<(unsigned)c.M, 256, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace dptq
