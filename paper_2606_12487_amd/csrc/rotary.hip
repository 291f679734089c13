// Rotary positions on queries and keys [T, heads, D] in one launch (the
// mathematics: rotary_device.h).
//
// A wave takes one token and up to 64 N units of its heads (a unit: eight pairs,
// two 16-byte loads and stores).  It computes the token's angles once, a lane
// each, into LDS, and every head reads them there.
//
// Bound by bytes: 4099 tokens of 64 + 8 heads of 128 take 33 us, 4.6 TB/s.  Loads and
// stores that do not stay in the caches take 29.5 us, but between a producer of the
// rows and a reader of the result nothing is left of it (4099 tokens 78.4 for 78.7 us
// of all three, 2048 tokens 39.7 for 37.9).
#include "internal.h"
#include "rotary_device.h"

namespace dptq {
namespace {

constexpr int kWaves = 4;

struct RotaryArgs {
  Rotary r;
  const __half *q, *k;
  __half *q_out, *k_out;
  int64_t ld_q, ld_k, ld_q_out, ld_k_out;
  int heads, kv_heads, parts;   // parts: waves of a token
  int64_t waves;                // of the launch
  const int32_t* positions;
};

template <bool INTER, bool WIDE, int N>
__global__ void __launch_bounds__(kWaves * 64) rotary_kernel(RotaryArgs a) {
  __shared__ float2 angles[kWaves][kMaxRotaryHead / 2];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t item = (int64_t)blockIdx.x * kWaves + wave;
  if (item >= a.waves) return;
  const int token = (int)(item / a.parts), part = (int)(item - (int64_t)token * a.parts);
  rotary_angles(a.r, a.positions[token], angles[wave], lane);
  const RotaryRows q{a.q + token * a.ld_q, a.q_out + token * a.ld_q_out, a.heads};
  const RotaryRows k{a.k + token * a.ld_k, a.k_out + token * a.ld_k_out, a.kv_heads};
  rotary_units<INTER, WIDE, N>(a.r, angles[wave], q, k, part * 64 * N, lane);
}

template <int N>
void launch_n(const RotaryArgs& a, hipStream_t stream) {
  const unsigned grid = (unsigned)((a.waves + kWaves - 1) / kWaves);
  if (a.r.interleaved)
    a.r.wide ? rotary_kernel<true, true, N><<<grid, kWaves * 64, 0, stream>>>(a)
             : rotary_kernel<true, false, N><<<grid, kWaves * 64, 0, stream>>>(a);
  else
    a.r.wide ? rotary_kernel<false, true, N><<<grid, kWaves * 64, 0, stream>>>(a)
             : rotary_kernel<false, false, N><<<grid, kWaves * 64, 0, stream>>>(a);
}

}  // namespace

Rotary make_rotary(const double* inv_freq, int D, int rotary_dim, bool interleaved, float scale) {
  Rotary r{};
  r.inv_freq = inv_freq;
  r.D = D;
  r.half = rotary_dim / 2;
  r.scale = scale;
  r.interleaved = interleaved;
  r.wide = rotary_dim % (interleaved ? 8 : 16) == 0;
  r.units = !r.wide ? D - r.half : interleaved ? D / 8 : (D - r.half) / 8;
  r.units_inv = r.units > 1 ? (uint32_t)((((uint64_t)1 << 32) + r.units - 1) / r.units) : 0u;
  return r;
}

hipError_t launch_rotary(const RotaryCall& c, hipStream_t stream) {
  RotaryArgs a{};
  a.r = make_rotary(c.inv_freq, c.head_dim, c.rotary_dim, c.interleaved, c.scale);
  a.q = static_cast<const __half*>(c.q);
  a.k = static_cast<const __half*>(c.k);
  a.q_out = static_cast<__half*>(c.q_out);
  a.k_out = static_cast<__half*>(c.k_out);
  a.ld_q = c.ld_q;
  a.ld_k = c.ld_k;
  a.ld_q_out = c.ld_q_out;
  a.ld_k_out = c.ld_k_out;
  a.heads = c.heads;
  a.kv_heads = c.kv_heads;
  a.positions = c.positions;
  const int64_t units = (int64_t)(c.heads + c.kv_heads) * a.r.units;
  const bool few = c.T * units < (int64_t)device_cus() * 4 * 64 * 4;
  a.parts = (int)((units + (few ? 63 : 255)) / (few ? 64 : 256));
  // A launch holds less than 2^32 threads.
  const int64_t most = 0xFFFFFFFFll / 64 / a.parts - kWaves;
  for (int64_t t = 0; t < c.T; t += most) {
    a.waves = (c.T - t < most ? c.T - t : most) * a.parts;
    if (few) launch_n<1>(a, stream);
    else launch_n<4>(a, stream);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    a.positions += most;
    a.q += most * c.ld_q;
    a.q_out += most * c.ld_q_out;
    if (c.kv_heads > 0) {
      a.k += most * c.ld_k;
      a.k_out += most * c.ld_k_out;
    }
  }
  return hipSuccess;
}

}  // namespace dptq
