// Residual addition, root-mean-square norm and 8-bit codes of each row:
//
//   h = fl16(x + residual)                  (h = x without a residual)
//   t_k = h_k * w_k                         (exact: two fp16 factors in fp32)
//   s = fl32(max|t| / 127),  code_k = RNE(fl32(t_k / s))      (0 where s = 0)
//   scale = fl32(s * r),     r = 1 / sqrt(sum(h^2) / K + eps)
//
// so that code * scale is the normalised row r * h * w in 8 bits.  r is common
// to a row and cancels out of t / s: the codes depend on no sum and on no
// order of summation.
//
// One workgroup a row, the row held in registers between the reduction and the
// codes: x, the residual and the weight are read once, h and the codes written
// once.  Bound by those 7 bytes an element: 4001 rows of 8192 take 44.6 us, 5.15
// TB/s, as a large copy does; one row of 4096 takes 3 us, a launch.
#include "internal.h"
#include "wave_device.h"

namespace dptq {
namespace {

struct Row8 {   // eight halves
  uint32_t w[4];
};

__device__ __forceinline__ float lo_half(uint32_t w) {
  return __half2float(__ushort_as_half((unsigned short)(w & 0xFFFFu)));
}
__device__ __forceinline__ float hi_half(uint32_t w) {
  return __half2float(__ushort_as_half((unsigned short)(w >> 16)));
}
__device__ __forceinline__ uint32_t pack_halves(float a, float b) {
  return (uint32_t)__half_as_ushort(__float2half_rn(a)) | ((uint32_t)__half_as_ushort(__float2half_rn(b)) << 16);
}
__device__ __forceinline__ Row8 load8(const uint4* p) {
  const uint4 v = *p;
  return Row8{{v.x, v.y, v.z, v.w}};
}

// fl32(t / s) from rc = fl32(1 / s): the residual t - q s is exact under an
// FMA, and the corrected quotient is the correctly rounded one.  Rounded to an
// integer by the fp32 adder.
__device__ __forceinline__ uint32_t code8(float t, float s, float rc) {
  const float q = t * rc;
  const float e = fmaf(-q, s, t);
  const float u = fmaf(e, rc, q) + 12582912.0f;   // 1.5 * 2^23
  return __float_as_uint(u) & 0xFFu;
}

template <int THREADS, int VPT>
__global__ void __launch_bounds__(THREADS)
rms_norm_quant_kernel(const uint4* x, const uint4* residual, const uint4* __restrict__ weight, int64_t M,
                      int n8, float inv_k, float eps, uint4* sum, uint2* __restrict__ codes,
                      float* __restrict__ scales) {
  __shared__ float2 part[THREADS / 64];
  for (int64_t row = blockIdx.x; row < M; row += gridDim.x) {
    const int64_t base = row * n8;
    Row8 h[VPT];
    float sq = 0.0f, top = 0.0f;
#pragma unroll
    for (int v = 0; v < VPT; ++v) {
      const int c = (int)threadIdx.x + v * THREADS;
      h[v] = Row8{{0, 0, 0, 0}};
      if (c < n8) {
        h[v] = load8(x + base + c);
        if (residual) {
          const Row8 r = load8(residual + base + c);
#pragma unroll
          for (int i = 0; i < 4; ++i)
            h[v].w[i] = pack_halves(lo_half(h[v].w[i]) + lo_half(r.w[i]), hi_half(h[v].w[i]) + hi_half(r.w[i]));
          sum[base + c] = make_uint4(h[v].w[0], h[v].w[1], h[v].w[2], h[v].w[3]);
        }
        const Row8 w = load8(weight + c);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float a = lo_half(h[v].w[i]), b = hi_half(h[v].w[i]);
          sq = fmaf(a, a, sq);
          sq = fmaf(b, b, sq);
          top = fmaxf(top, fmaxf(fabsf(a * lo_half(w.w[i])), fabsf(b * hi_half(w.w[i]))));
        }
      }
    }
    sq = wave_sum(sq);
    top = wave_max(top);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x / 64] = make_float2(sq, top);
    __syncthreads();
    sq = 0.0f;
#pragma unroll
    for (int i = 0; i < THREADS / 64; ++i) {
      sq += part[i].x;
      top = fmaxf(top, part[i].y);
    }
    const float s = top / 127.0f;
    const float rc = s > 0.0f ? 1.0f / s : 0.0f;   // a row of zeros: codes 0
#pragma unroll
    for (int v = 0; v < VPT; ++v) {
      const int c = (int)threadIdx.x + v * THREADS;
      if (c < n8) {
        const Row8 w = load8(weight + c);
        uint32_t out[2] = {0, 0};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          out[i / 2] |= code8(lo_half(h[v].w[i]) * lo_half(w.w[i]), s, rc) << (16 * (i & 1));
          out[i / 2] |= code8(hi_half(h[v].w[i]) * hi_half(w.w[i]), s, rc) << (16 * (i & 1) + 8);
        }
        codes[base + c] = make_uint2(out[0], out[1]);
      }
    }
    if (threadIdx.x == 0) scales[row] = s > 0.0f ? s * (1.0f / sqrtf(sq * inv_k + eps)) : 0.0f;
    __syncthreads();   // part is free again
  }
}

template <int THREADS, int VPT>
hipError_t launch(const void* x, const void* residual, const void* weight, int64_t M, int K, float eps,
                  void* sum, int8_t* codes, float* scales, hipStream_t stream) {
  const unsigned grid = (unsigned)(M < 1 << 20 ? M : 1 << 20);
  rms_norm_quant_kernel<THREADS, VPT><<<grid, THREADS, 0, stream>>>(
      static_cast<const uint4*>(x), static_cast<const uint4*>(residual), static_cast<const uint4*>(weight), M,
      K / 8, 1.0f / (float)K, eps, static_cast<uint4*>(sum), reinterpret_cast<uint2*>(codes), scales);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rms_norm_quant(const void* x, const void* residual, const void* weight, int64_t M, int K,
                                 float eps, void* sum, int8_t* codes, float* scales, hipStream_t stream) {
  const int n8 = K / 8;
  if (n8 <= 256) return launch<256, 1>(x, residual, weight, M, K, eps, sum, codes, scales, stream);
  if (n8 <= 1024) return launch<256, 4>(x, residual, weight, M, K, eps, sum, codes, scales, stream);
  if (n8 <= 4096) return launch<1024, 4>(x, residual, weight, M, K, eps, sum, codes, scales, stream);
  return launch<1024, 8>(x, residual, weight, M, K, eps, sum, codes, scales, stream);
}

}  // namespace dptq
