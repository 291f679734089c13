// Reductions over the 64 lanes of a wavefront in the vector ALU: lane exchanges
// within rows of 16 by DPP, between rows by the permlane swaps (six steps; the
// same exchanges through LDS, as __shfl_xor makes them, take a few times as
// long, which is what a kernel of one short reduction consists of).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace dptq {

template <int CTRL>
__device__ __forceinline__ float dpp(float x) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xF, 0xF, true));
}

// op over all lanes, the result in each; op must commute.
template <typename Op>
__device__ __forceinline__ float wave_reduce(float x, Op op) {
  x = op(x, dpp<0xB1>(x));    // quad_perm 1, 0, 3, 2
  x = op(x, dpp<0x4E>(x));    // quad_perm 2, 3, 0, 1
  x = op(x, dpp<0x141>(x));   // row_half_mirror: the other quad of eight
  x = op(x, dpp<0x140>(x));   // row_mirror: the other half of a row
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = op(__uint_as_float(r[0]), __uint_as_float(r[1]));
  const auto h = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return op(__uint_as_float(h[0]), __uint_as_float(h[1]));
}
__device__ __forceinline__ float wave_max(float x) {
  return wave_reduce(x, [](float a, float b) { return fmaxf(a, b); });
}
__device__ __forceinline__ float wave_sum(float x) {
  return wave_reduce(x, [](float a, float b) { return a + b; });
}

}  // namespace dptq
