// Rotary positions on rows of fp16 heads, shared by the kernel that only
// rotates (rotary.hip) and the one that writes the cache too
// (kv8_rotary_append.hip).
//
// Pair i of the first r = 2 half channels of a head, channels (i, i + half) or,
// interleaved, (2i, 2i + 1), turns by the angle position * inv_freq[i]:
//
//   y1 = fl16(x1 c - x2 s),  y2 = fl16(x1 s + x2 c),  (c, s) = scale * (cos, sin)
//
// The angle is a product in 64 bits (a position of 2^20 in 32 bits would be off
// by 2^-4 rad) of which only the part within a quarter turn goes on in 32 bits:
// (c, s) are off by a few roundings of 2^-24, below 2^-21, which the rounding of
// the result to fp16, 2^-11, makes hardly different from 64-bit cosines.
#pragma once

#include <hip/hip_runtime.h>
#include <hip/hip_fp16.h>
#include <stdint.h>

namespace dptq {

constexpr int kMaxRotaryHead = 512;   // channels of a head

struct Rotary {
  const double* inv_freq;   // [half]
  int D, half;
  float scale;
  bool interleaved;
  bool wide;                // the pairs' octets of channels are whole: 16-byte loads
  int units;                // of a head: an octet of pairs (wide) or a pair, and what is only copied
  uint32_t units_inv;       // ceil(2^32 / units); 0 for one unit
};
// rotary_dim even, at most D; D a multiple of 8, at most kMaxRotaryHead (rotary.hip).
Rotary make_rotary(const double* inv_freq, int D, int rotary_dim, bool interleaved, float scale);

// scale * (cos, sin) of p * f.
__device__ __forceinline__ float2 rotary_angle(int p, double f, float scale) {
  constexpr double kTurns = 0.15915494309189533577;   // 1 / (2 pi)
  const double t = ((double)p * f) * kTurns;
  const double q4 = 4.0 * (t - __builtin_rint(t));    // quarter turns, [-2, 2]
  const double k = __builtin_rint(q4);
  // |x| <= pi / 4: the series' next terms are below 2^-29 (sine) and 2^-32.
  const float x = (float)(q4 - k) * 1.57079632679489662f;
  const float z = x * x;
  float s = __builtin_fmaf(z, 2.7557319e-6f, -1.9841270e-4f);
  s = __builtin_fmaf(z, s, 8.3333333e-3f);
  s = __builtin_fmaf(z, s, -0.16666667f);
  s = __builtin_fmaf(x * z, s, x);
  float c = __builtin_fmaf(z, -2.7557319e-7f, 2.4801587e-5f);
  c = __builtin_fmaf(z, c, -1.3888889e-3f);
  c = __builtin_fmaf(z, c, 4.1666667e-2f);
  c = __builtin_fmaf(z, c, -0.5f);
  c = __builtin_fmaf(z, c, 1.0f);
  const int quadrant = (int)k;                        // -2 .. 2
  const float a = quadrant & 1 ? s : c, b = quadrant & 1 ? c : s;   // |cos|, |sin|
  return make_float2(scale * ((quadrant + 1) & 2 ? -a : a), scale * (quadrant & 2 ? -b : b));
}

// i / n for i n < 2^32, with inv = ceil(2^32 / n), 0 for n = 1.
__device__ __forceinline__ int rotary_divide(int i, uint32_t inv) {
  return inv ? (int)__umulhi((uint32_t)i, inv) : i;
}

// The empty asm keeps a result an fp32 value: the backend may fold an FMA and the
// conversion to fp16 behind it into one rounding, in one kernel and not in
// another, and every kernel here has to give the same bits.
__device__ __forceinline__ float rotary_first(float a, float b, float2 cs) {
  float y = __builtin_fmaf(a, cs.x, -(b * cs.y));
  asm("" : "+v"(y));
  return y;
}
__device__ __forceinline__ float rotary_second(float a, float b, float2 cs) {
  float y = __builtin_fmaf(a, cs.y, b * cs.x);
  asm("" : "+v"(y));
  return y;
}

__device__ __forceinline__ void unpack8(uint4 v, float* f) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const __half2 h = *reinterpret_cast<const __half2*>(&w[j]);
    f[2 * j] = __low2float(h);
    f[2 * j + 1] = __high2float(h);
  }
}
__device__ __forceinline__ uint4 pack8(const float* f) {
  uint32_t w[4];
#pragma unroll
  for (int j = 0; j < 4; ++j)
    w[j] = (uint32_t)__half_as_ushort(__float2half_rn(f[2 * j])) |
           ((uint32_t)__half_as_ushort(__float2half_rn(f[2 * j + 1])) << 16);
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// A token's rows of one tensor: head 0 of the input and of the output.
struct RotaryRows {
  const __half* x;
  __half* out;
  int heads;
};

// The angles of a token at position p, by the lanes of one wave, into its cs.
__device__ __forceinline__ void rotary_angles(const Rotary& r, int p, float2* cs, int lane) {
  for (int i = lane; i < r.half; i += 64) cs[i] = rotary_angle(p, r.inv_freq[i], r.scale);
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// Units [first, first + 64 N) of a token's heads, those of a before those of b,
// by the lanes of one wave.
template <bool INTER, bool WIDE, int N>
__device__ __forceinline__ void rotary_units(const Rotary& r, const float2* cs, const RotaryRows& a,
                                             const RotaryRows& b, int first, int lane) {
  const int total = (a.heads + b.heads) * r.units;
  const __half* from[N];
  __half* to[N];
  int unit[N];
#pragma unroll
  for (int n = 0; n < N; ++n) {
    const int i = first + 64 * n + lane;
    const int h = rotary_divide(i, r.units_inv);
    unit[n] = i < total ? i - h * r.units : -1;
    const bool second = h >= a.heads;
    const int64_t at = (int64_t)(second ? h - a.heads : h) * r.D;
    from[n] = (second ? b.x : a.x) + at;
    to[n] = (second ? b.out : a.out) + at;
  }
  if constexpr (WIDE) {
    const int pairs = INTER ? r.half / 4 : r.half / 8;   // units that turn
    uint4 v[N], w[N];
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const int u = unit[n];
      if (u < 0) continue;
      // The channels behind the pairs follow in octets.
      v[n] = *reinterpret_cast<const uint4*>(from[n] + (INTER || u < pairs ? 8 * u : 2 * r.half + 8 * (u - pairs)));
      if (!INTER && u < pairs) w[n] = *reinterpret_cast<const uint4*>(from[n] + r.half + 8 * u);
    }
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const int u = unit[n];
      if (u < 0) continue;
      if (u >= pairs) {
        if (to[n] != from[n])
          *reinterpret_cast<uint4*>(to[n] + (INTER ? 8 * u : 2 * r.half + 8 * (u - pairs))) = v[n];
        continue;
      }
      float f[8], y[8];
      unpack8(v[n], f);
      if constexpr (INTER) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float2 t = cs[4 * u + j];
          y[2 * j] = rotary_first(f[2 * j], f[2 * j + 1], t);
          y[2 * j + 1] = rotary_second(f[2 * j], f[2 * j + 1], t);
        }
        *reinterpret_cast<uint4*>(to[n] + 8 * u) = pack8(y);
      } else {
        float g[8], z[8];
        unpack8(w[n], g);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float2 t = cs[8 * u + j];
          y[j] = rotary_first(f[j], g[j], t);
          z[j] = rotary_second(f[j], g[j], t);
        }
        *reinterpret_cast<uint4*>(to[n] + 8 * u) = pack8(y);
        *reinterpret_cast<uint4*>(to[n] + r.half + 8 * u) = pack8(z);
      }
    }
  } else {
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const int u = unit[n];
      if (u < 0) continue;
      if (u >= r.half) {
        if (to[n] != from[n]) to[n][r.half + u] = from[n][r.half + u];
        continue;
      }
      const int c1 = INTER ? 2 * u : u, c2 = INTER ? 2 * u + 1 : u + r.half;
      const float f = __half2float(from[n][c1]), g = __half2float(from[n][c2]);
      to[n][c1] = __float2half_rn(rotary_first(f, g, cs[u]));
      to[n][c2] = __float2half_rn(rotary_second(f, g, cs[u]));
    }
  }
}

}  // namespace dptq
