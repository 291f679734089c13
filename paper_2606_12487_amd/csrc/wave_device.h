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

// Sums over the lanes up to each, in the vector ALU; exact for integers.
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t dpp_or_0(uint32_t x) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, ROWS, 0xF, false);
}
template <int CTRL, int ROWS>
__device__ __forceinline__ unsigned long long dpp_or_0(unsigned long long x) {
  return (unsigned long long)dpp_or_0<CTRL, ROWS>((uint32_t)(x >> 32)) << 32 | dpp_or_0<CTRL, ROWS>((uint32_t)x);
}
template <typename V>
__device__ __forceinline__ V wave_scan(V x) {
  x += dpp_or_0<0x111, 0xF>(x);   // row_shr 1, 2, 4, 8: within rows of 16
  x += dpp_or_0<0x112, 0xF>(x);
  x += dpp_or_0<0x114, 0xF>(x);
  x += dpp_or_0<0x118, 0xF>(x);
  x += dpp_or_0<0x142, 0xA>(x);   // lane 15 of a row to the next, into rows 1 and 3
  x += dpp_or_0<0x143, 0xC>(x);   // lane 31 to the upper half
  return x;
}

// The value of lane ^ J.
template <int J>
__device__ __forceinline__ uint32_t lane_xor(uint32_t x) {
  static_assert(J == 1 || J == 2 || J == 4 || J == 8 || J == 16 || J == 32);
  const int v = (int)x;
  if constexpr (J == 1) return (uint32_t)__builtin_amdgcn_update_dpp(v, v, 0xB1, 0xF, 0xF, true);
  if constexpr (J == 2) return (uint32_t)__builtin_amdgcn_update_dpp(v, v, 0x4E, 0xF, 0xF, true);
  if constexpr (J == 4) {   // the mirror of eight, of which each quad is mirrored back
    const int m = __builtin_amdgcn_update_dpp(v, v, 0x141, 0xF, 0xF, true);
    return (uint32_t)__builtin_amdgcn_update_dpp(m, m, 0x1B, 0xF, 0xF, true);
  }
  if constexpr (J == 8) return (uint32_t)__builtin_amdgcn_update_dpp(v, v, 0x128, 0xF, 0xF, true);   // row_ror 8
  if constexpr (J == 16) {
    const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    return threadIdx.x & 16 ? r[0] : r[1];
  }
  if constexpr (J == 32) {
    const auto r = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    return threadIdx.x & 32 ? r[0] : r[1];
  }
}

}  // namespace dptq
