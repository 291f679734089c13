// What the kernels share that write the 8-bit paged cache (layout: kv8_device.h):
// kv8_append.hip and kv8_rotary_append.hip.
#pragma once

#include "internal.h"
#include "kv8_device.h"

namespace dptq {

struct AppendArgs {
  const __half* x[2];   // K, V rows
  int64_t ld[2];
  uint8_t* pages[2];
  float* scales[2];
  const int32_t *cu, *lengths, *table;
  int T, max_pages, num_pages, heads;
};

inline AppendArgs append_args(const Kv8Cache& c, const void* k, int64_t ld_k, const void* v, int64_t ld_v) {
  AppendArgs a{};
  a.x[0] = static_cast<const __half*>(k);
  a.x[1] = static_cast<const __half*>(v);
  a.ld[0] = ld_k;
  a.ld[1] = ld_v;
  a.pages[0] = c.k_pages;
  a.pages[1] = c.v_pages;
  a.scales[0] = c.k_scales;
  a.scales[1] = c.v_scales;
  a.cu = c.cu;
  a.lengths = c.lengths;
  a.table = c.table;
  a.T = (int)c.T;
  a.max_pages = (int)c.max_pages;
  a.num_pages = (int)c.num_pages;
  a.heads = c.kv_heads;
  return a;
}

// Two floats to e4m3, in the low or high half of old.
template <bool HI>
__device__ __forceinline__ uint32_t to_e4m3(float a, float b, uint32_t old) {
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(a, b, (int)old, HI);
}

__device__ __forceinline__ uint32_t rescale4(uint32_t c, float ratio) {
  const uint32_t lo = to_e4m3<false>(__builtin_amdgcn_cvt_f32_fp8((int)c, 0) * ratio,
                                     __builtin_amdgcn_cvt_f32_fp8((int)c, 1) * ratio, 0);
  return to_e4m3<true>(__builtin_amdgcn_cvt_f32_fp8((int)c, 2) * ratio,
                       __builtin_amdgcn_cvt_f32_fp8((int)c, 3) * ratio, lo);
}

// Exponent of the scale for a largest magnitude a (448 = 1.75 * 2^8).
__device__ __forceinline__ int scale_exp(float a) {
  const uint32_t u = __float_as_uint(a);
  const int e = (int)(u >> 23) - 127 - 8 + ((u & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  return max(e, kKv8MinExp);
}

// Bytes of the dword of slots [first, first + 4) that lie in [lo, hi).
__device__ __forceinline__ uint32_t slot_mask(int first, int lo, int hi) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (first + i >= lo && first + i < hi) m |= 0xFFu << (8 * i);
  return m;
}

}  // namespace dptq
