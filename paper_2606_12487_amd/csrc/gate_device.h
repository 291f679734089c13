// The epilogue of a gated feed-forward block, for every GEMM kernel: of the
// dequantized values g of a gate channel and u of the up channel beside it
//
//   y = fl16(g * sigmoid(t(g)) * u),  t(g) = g (SiLU) or
//   2 sqrt(2 / pi) (g + 0.044715 g^3) (GELU in its tanh form)
//
// in fp32, without a rounding of g and u to fp16 in between.  Weight rows 16 i to
// 16 i + 7 are the gate channels 8 i to 8 i + 7 and the eight rows behind them the
// same up channels, so that with 32 x 32 accumulators both values are in one lane
// and with 16 x 16 ones half a wavefront apart, on every tile of 16 rows.
#pragma once

#include <hip/hip_runtime.h>
#include <hip/hip_fp16.h>
#include <stdint.h>

namespace dptq {

// -t(g) log2(e) = g (k1 + k2 g^2).
struct Gate {
  float k1, k2;
};

// u g / (1 + exp(-t)).  exp2 and the reciprocal are the hardware's, each within one
// unit in the last place of 32 bits, 2^-23, beside a rounding of 2^-11 to fp16: a
// division and an exp in full would lengthen an epilogue that the matrix pipes wait
// for.  Where exp overflows the quotient is 0, as it should be (g is finite); g^2 is
// kept finite for k2 = 0.
__device__ __forceinline__ __half gated(float g, float u, Gate k) {
  const float t = g * __builtin_fmaf(k.k2, fminf(g * g, 3.0e38f), k.k1);
  float y = (g * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(t))) * u;
  asm("" : "+v"(y));   // an fp32 value, as the plain epilogue's
  return __float2half_rn(y);
}

// Four channels: their accumulators, as fp32 values, and scales.
__device__ __forceinline__ uint2 gated4(float4 g, float4 u, float as, float4 wg, float4 wu, Gate k) {
  const __half h0 = gated((g.x * as) * wg.x, (u.x * as) * wu.x, k), h1 = gated((g.y * as) * wg.y, (u.y * as) * wu.y, k);
  const __half h2 = gated((g.z * as) * wg.z, (u.z * as) * wu.z, k), h3 = gated((g.w * as) * wg.w, (u.w * as) * wu.w, k);
  return make_uint2((uint32_t)__half_as_ushort(h0) | ((uint32_t)__half_as_ushort(h1) << 16),
                    (uint32_t)__half_as_ushort(h2) | ((uint32_t)__half_as_ushort(h3) << 16));
}

}  // namespace dptq
