// Rotary positions and the 8-bit cache's append in one launch: the new tokens'
// queries rotated into another tensor, their keys rotated and rounded to fp16 and
// their values written into the cache, with the bits of rotary and kv8_append one
// after the other (the mathematics: rotary_device.h, kv8_append.hip).
//
// Workgroups of three kinds.  One of K or V takes a page that new tokens of a
// sequence fall into and a head: the page's rows, rotated for K, go through LDS
// while the page's scale is found, and out again as codes, for V by channels.  One
// of the queries takes tokens and parts of their heads, each a wave's.
//
// The queries are bound by bytes, the pages by their chain of loads (offsets,
// table, rows), and both by how many of them are resident: loops that are not
// unrolled keep it to 125 registers at every head size, four workgroups a CU.  With
// a page's rows in registers instead, as kv8_append.hip has them, 256 channels had
// one: 2 x 1000 tokens of 32 + 32 heads of 256 took 60 us for 38, 32 x 152 of 16 +
// 16 of 64 35 for 28.  Five workgroups (launch bounds) spill.
//
// 4500 tokens of three prompts, 64 + 8 heads of 128: 41 us, 4.1 TB/s (rotary alone
// 33 for 4099 tokens); 64 single tokens: 9.5.
#include "internal.h"
#include "kv8_write.h"
#include "rotary_device.h"
#include "wave_device.h"

namespace dptq {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kRotaryUnits = 4;   // of a lane

// The queries' side.
struct RotaryQ {
  Rotary r;
  const __half* q;
  __half* out;
  int64_t ld, ld_out;
  int heads, parts;   // parts of 64 kRotaryUnits units
};

// Rotates the queries of tokens [64 x, 64 x + 64) of a sequence, and so on by
// gridDim.x; the workgroup is slice `slice` of `slices` of them.
template <bool INTER, bool WIDE>
__device__ __forceinline__ void rotate_q(const RotaryQ& a, const KvSeq& s, int slice, int slices, float2* angles) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  for (int64_t first = 64 * (int64_t)blockIdx.x; first < s.count; first += 64 * (int64_t)gridDim.x) {
    const int tokens = (int)min((int64_t)64, s.count - first);
    for (int i = slice * kWaves + wave; i < tokens * a.parts; i += slices * kWaves) {
      const int t = i / a.parts, part = i - t * a.parts;
      const int64_t row = s.first_row + first + t;
      rotary_angles(a.r, (int)(s.start + first + t), angles, lane);
      rotary_units<INTER, WIDE, kRotaryUnits>(a.r, angles, RotaryRows{a.q + row * a.ld, a.out + row * a.ld_out, a.heads},
                                              RotaryRows{nullptr, nullptr, 0}, part * 64 * kRotaryUnits, lane);
      // The next token's angles wait for these reads.
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
      __builtin_amdgcn_wave_barrier();
    }
  }
}

// Octet v (channels c to c + 7) of the key row at head, of the token at position
// p, rotated; freq: the frequencies of its channels.
__device__ __forceinline__ uint4 rotate_octet(const Rotary& r, uint4 v, const __half* head, int c, int p,
                                              const double (&freq)[8]) {
  if (c >= 2 * r.half) return v;
  float f[8], g[8], y[8];
  unpack8(v, f);
  if (r.interleaved) {
#pragma unroll
    for (int j = 0; j < 8; j += 2) {
      y[j] = f[j];
      y[j + 1] = f[j + 1];
      if (c + j >= 2 * r.half) continue;   // an octet that the pairs end in
      const float2 t = rotary_angle(p, freq[j], r.scale);
      y[j] = rotary_first(f[j], f[j + 1], t);
      y[j + 1] = rotary_second(f[j], f[j + 1], t);
      __builtin_amdgcn_sched_barrier(0);   // one angle at a time: registers
    }
    return pack8(y);
  }
  if (r.wide) {
    unpack8(*reinterpret_cast<const uint4*>(head + (c >= r.half ? c - r.half : c + r.half)), g);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int ch = c + j;
      if (ch < 2 * r.half) g[j] = __half2float(head[ch < r.half ? ch + r.half : ch - r.half]);
    }
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const int ch = c + j;
    y[j] = f[j];
    if (ch >= 2 * r.half) continue;
    const float2 t = rotary_angle(p, freq[j], r.scale);
    y[j] = ch >= r.half ? rotary_second(g[j], f[j], t) : rotary_first(f[j], g[j], t);
    __builtin_amdgcn_sched_barrier(0);
  }
  return pack8(y);
}

template <int D>
__global__ void __launch_bounds__(kThreads) rotary_append_kernel(AppendArgs a, RotaryQ rq) {
  constexpr int kOctets = D / 8;               // of channels
  constexpr int kStep = kThreads / kOctets;    // slots that the threads' octets cover at a time
  // The page's rows, an octet of slot s at s * kOctets + (octet ^ turn(s)); or a
  // token's angles in each wave.
  __shared__ uint4 stage[kPage * kOctets];
  __shared__ float part[kWaves];
  const int b = blockIdx.z, tid = threadIdx.x;
  const KvSeq q = kv_seq(a.cu, a.lengths, b, a.T);
  if ((int)blockIdx.y >= 2 * a.heads) {
    float2* const mine = reinterpret_cast<float2*>(stage) + (tid >> 6) * (D / 2);
    const int slice = (int)blockIdx.y - 2 * a.heads, slices = (int)gridDim.y - 2 * a.heads;
    if (rq.r.interleaved)
      rq.r.wide ? rotate_q<true, true>(rq, q, slice, slices, mine) : rotate_q<true, false>(rq, q, slice, slices, mine);
    else
      rq.r.wide ? rotate_q<false, true>(rq, q, slice, slices, mine) : rotate_q<false, false>(rq, q, slice, slices, mine);
    return;
  }
  if (q.count == 0 || q.length == 0) return;
  const int head = (int)blockIdx.y >> 1;
  const bool is_v = blockIdx.y & 1;
  const int octet = tid % kOctets, c = 8 * octet;
  // The frequencies of the octet's channels, ahead of the table and the rows.
  double freq[8] = {};
  if (!is_v) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int ch = c + j;
      const int pair = rq.r.interleaved ? ch >> 1 : ch >= rq.r.half ? ch - rq.r.half : ch;
      if (ch < 2 * rq.r.half) freq[j] = rq.r.inv_freq[pair];
    }
  }
  const int begin = max(q.start, 0);
  const int last_block = min((q.length - 1) / kPage, a.max_pages - 1);
  for (int blk = begin / kPage + blockIdx.x; blk <= last_block; blk += gridDim.x) {
    const int page = a.table[(int64_t)b * a.max_pages + blk];
    if ((uint32_t)page >= (uint32_t)a.num_pages) continue;
    const int lo = max(begin - blk * kPage, 0);                    // new slots [lo, hi)
    const int hi = min(q.length - blk * kPage, kPage);
    const bool fresh = lo == 0;
    const int64_t at = (int64_t)page * a.heads + head;
    uint8_t* const codes = a.pages[is_v] + at * (kPage * D);
    const float had = fresh ? 0.0f : a.scales[is_v][at];

    // The new tokens' rows into LDS, and their largest magnitude.  V's octets are
    // turned by the slot's eighth, for the reads by channels below: the 64 lanes
    // then read 32 dwords of as many banks.
    float top = 0.0f;
    const __half* const row0 = a.x[is_v] + (int64_t)head * D;
#pragma unroll 1
    for (int first = lo / kStep * kStep; first < hi; first += kStep) {
      const int slot = first + tid / kOctets;
      if (slot < lo || slot >= hi) continue;
      const int p = blk * kPage + slot;
      const __half* const row = row0 + ((int64_t)q.first_row + ((int64_t)p - q.start)) * a.ld[is_v];
      uint4 v = *reinterpret_cast<const uint4*>(row + c);
      if (!is_v) v = rotate_octet(rq.r, v, row, c, p, freq);
      float f[8];
      unpack8(v, f);
#pragma unroll
      for (int j = 0; j < 8; ++j) top = fmaxf(top, fabsf(f[j]));
      stage[slot * kOctets + (is_v ? octet ^ (slot >> 3) : octet)] = v;
    }
    top = wave_max(top);
    if ((tid & 63) == 0) part[tid / 64] = top;
    __syncthreads();   // and everyone has read the scale
#pragma unroll
    for (int i = 0; i < kWaves; ++i) top = fmaxf(top, part[i]);
    const float s = fmaxf(__uint_as_float((uint32_t)(scale_exp(top) + 127) << 23), had);
    const bool grew = !fresh && s > had;
    const float ratio = had / s, inv = 1.0f / s;   // exact for powers of two
    if (tid == 0) a.scales[is_v][at] = s;

    if (!is_v) {
      // New slots; those before them where the scale grew, those behind them where
      // the page is new.
#pragma unroll 1
      for (int first = grew ? 0 : lo / kStep * kStep; first < (fresh ? kPage : hi); first += kStep) {
        const int slot = first + tid / kOctets;
        uint2* const dst = reinterpret_cast<uint2*>(codes + slot * D + c);
        if (slot >= lo && slot < hi) {
          float f[8];
          unpack8(stage[slot * kOctets + octet], f);
#pragma unroll
          for (int j = 0; j < 8; ++j) f[j] *= inv;
          *dst = make_uint2(to_e4m3<true>(f[2], f[3], to_e4m3<false>(f[0], f[1], 0)),
                            to_e4m3<true>(f[6], f[7], to_e4m3<false>(f[4], f[5], 0)));
        } else if (slot >= hi) {
          if (fresh) *dst = make_uint2(0, 0);
        } else if (grew) {
          const uint2 o = *dst;
          *dst = make_uint2(rescale4(o.x, ratio), rescale4(o.y, ratio));
        }
      }
    } else {
      // Unit u: channel u / 8, slots 8 (u % 8) and up.
      const __half* const staged = reinterpret_cast<const __half*>(stage);
#pragma unroll 1
      for (int u = tid; u < 8 * D; u += kThreads) {
        const int d = u / 8, eighth = u % 8, first = 8 * eighth;
        uint8_t* const dst = codes + d * kPage + first;
        const bool any = first < hi && first + 8 > lo;
        if (!any && !fresh && !(grew && first < lo)) continue;
        float f[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int slot = first + j;
          const bool mine = slot >= lo && slot < hi;
          f[j] = mine ? __half2float(staged[(slot * kOctets + ((d >> 3) ^ eighth)) * 8 + (d & 7)]) * inv : 0.0f;
        }
        const uint2 n = make_uint2(to_e4m3<true>(f[2], f[3], to_e4m3<false>(f[0], f[1], 0)),
                                   to_e4m3<true>(f[6], f[7], to_e4m3<false>(f[4], f[5], 0)));
        if (fresh || (first >= lo && first + 8 <= hi)) {
          *reinterpret_cast<uint2*>(dst) = n;
        } else if (grew && first < lo) {
          const uint2 o = *reinterpret_cast<const uint2*>(dst);
          const uint32_t old0 = slot_mask(first, 0, lo), old1 = slot_mask(first + 4, 0, lo);
          const uint32_t new0 = slot_mask(first, lo, hi), new1 = slot_mask(first + 4, lo, hi);
          *reinterpret_cast<uint2*>(dst) =
              make_uint2((rescale4(o.x, ratio) & old0) | (n.x & new0) | (o.x & ~(old0 | new0)),
                         (rescale4(o.y, ratio) & old1) | (n.y & new1) | (o.y & ~(old1 | new1)));
        } else {
          // Single slots, without reading the page.
          for (int slot = max(lo, first); slot < min(hi, first + 8); ++slot)
            dst[slot - first] = (uint8_t)((slot - first < 4 ? n.x : n.y) >> (8 * ((slot - first) & 3)));
        }
      }
    }
    __syncthreads();   // part and stage are free again
  }
}

template <int D>
void launch(const AppendArgs& a, const RotaryQ& rq, dim3 grid, hipStream_t stream) {
  rotary_append_kernel<D><<<grid, kThreads, 0, stream>>>(a, rq);
}

}  // namespace

hipError_t launch_rotary_kv8_append(const Kv8Cache& c, const RotaryCall& r, const void* v, int64_t ld_v,
                                    int64_t max_new, hipStream_t stream) {
  AppendArgs a = append_args(c, r.k, r.ld_k, v, ld_v);
  if (c.num_pages == 0) a.max_pages = 0;   // nothing of the table is read
  RotaryQ rq{};
  rq.r = make_rotary(r.inv_freq, r.head_dim, r.rotary_dim, r.interleaved, r.scale);
  rq.q = static_cast<const __half*>(r.q);
  rq.out = static_cast<__half*>(r.q_out);
  rq.ld = r.ld_q;
  rq.ld_out = r.ld_q_out;
  rq.heads = r.heads;
  rq.parts = (int)(((int64_t)r.heads * rq.r.units + 64 * kRotaryUnits - 1) / (64 * kRotaryUnits));
  // A wave to each token and part; behind the pages' workgroups, whose chains of
  // loads are the longer ones (queries first: 46 us for 40, 4500 tokens).
  const int64_t waves = (max_new < 64 ? max_new : 64) * rq.parts;
  const int64_t slices = (waves + kWaves - 1) / kWaves;
  // Tiles of 64 tokens, and pages, that max_new tokens can touch; more loop.
  const int64_t tiles = (max_new + kPage - 2) / kPage + 1;
  const dim3 grid((unsigned)(tiles < 65535 ? tiles : 65535), (unsigned)(2 * c.kv_heads + (slices < 1024 ? slices : 1024)),
                  (unsigned)c.B);
  switch (c.head_dim) {
    case 64: launch<64>(a, rq, grid, stream); break;
    case 128: launch<128>(a, rq, grid, stream); break;
    case 256: launch<256>(a, rq, grid, stream); break;
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

}  // namespace dptq
