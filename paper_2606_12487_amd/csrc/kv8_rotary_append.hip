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
// table, rows) and by the angles, 64-bit products, and all by how many workgroups
// are resident: loops that are not unrolled and angles by way of LDS, a wave's lanes
// each a pair's, keep it to 80 registers, six workgroups a CU (four at 256
// channels).  Reading the next rows ahead costs eight registers more than it gains
// (256 single tokens of 32 + 8 heads: 14.5 us for 13).  Each key's octet with its own
// eight angles had 125 (4500 tokens of three prompts, 64 + 8 heads of 128: 41 us for
// 35); a page's rows in registers, as kv8_append.hip has them, one workgroup at 256
// channels (2 x 1000 tokens of 32 + 32 heads: 60 us for 38).  Dropped: four heads of
// 64 or two of 128 to a workgroup and its angles (39 us; 32 x 152 tokens of 16 + 16
// heads of 64 27 for 21): the chains take longer than the angles.
//
// 4500 tokens of three prompts: 37 us, 4.5 TB/s (35 to 38 on several cards; rotary
// alone 33 for 4099 tokens);
// 64 single tokens: 5.6 (9.5 with an octet's own angles, 7.6 with all eighths of V's
// page looked through for the one that changes).
#include "internal.h"
#include "kv8_write.h"
#include "rotary_device.h"
#include "wave_device.h"

namespace dptq {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kRotaryUnits = 2;   // of a lane

// The queries' side.
struct RotaryQ {
  Rotary r;
  const __half* q;
  __half* out;
  int64_t ld, ld_out;
  int heads, parts;    // parts of 64 kRotaryUnits units
  int run, pieces;     // parts that a wave turns by one token's angles, and such runs
};

// Rotates the queries of tokens [64 x, 64 x + 64) of a sequence, and so on by
// gridDim.x; the workgroup is slice `slice` of `slices` of them.
template <bool INTER, bool WIDE>
__device__ __forceinline__ void rotate_q(const RotaryQ& a, const KvSeq& s, int slice, int slices, float2* angles) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  for (int64_t first = 64 * (int64_t)blockIdx.x; first < s.count; first += 64 * (int64_t)gridDim.x) {
    const int tokens = (int)min((int64_t)64, s.count - first);
    for (int i = slice * kWaves + wave; i < tokens * a.pieces; i += slices * kWaves) {
      const int t = i / a.pieces, piece = i - t * a.pieces;
      const int64_t row = s.first_row + first + t;
      rotary_angles(a.r, (int)(s.start + first + t), angles, lane);
      const int end = min((piece + 1) * a.run, a.parts);
#pragma unroll 1
      for (int part = piece * a.run; part < end; ++part)
        rotary_units<INTER, WIDE, kRotaryUnits>(a.r, angles,
                                                RotaryRows{a.q + row * a.ld, a.out + row * a.ld_out, a.heads},
                                                RotaryRows{nullptr, nullptr, 0}, part * 64 * kRotaryUnits, lane);
      // The next token's angles wait for these reads.
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
      __builtin_amdgcn_wave_barrier();
    }
  }
}

// An octet of a key row, channels c to c + 7, and the octet of the other channels
// of its pairs, where these are one.
struct KeyOctet {
  uint4 v, other;
};
__device__ __forceinline__ KeyOctet key_octet(const Rotary& r, const __half* head, int c, bool rotated) {
  KeyOctet k;
  k.v = *reinterpret_cast<const uint4*>(head + c);
  if (rotated && r.wide && !r.interleaved && c < 2 * r.half)
    k.other = *reinterpret_cast<const uint4*>(head + (c >= r.half ? c - r.half : c + r.half));
  return k;
}

// The octet rotated, by its token's angles.
__device__ __forceinline__ uint4 rotate_octet(const Rotary& r, const KeyOctet& k, const __half* head, int c,
                                              const float2* angles) {
  if (c >= 2 * r.half) return k.v;
  float f[8], g[8], y[8];
  unpack8(k.v, f);
  if (r.interleaved) {
#pragma unroll
    for (int j = 0; j < 8; j += 2) {
      const float2 t = angles[(c + j) >> 1];
      const bool turns = c + j < 2 * r.half;   // the pairs may end in an octet
      y[j] = turns ? rotary_first(f[j], f[j + 1], t) : f[j];
      y[j + 1] = turns ? rotary_second(f[j], f[j + 1], t) : f[j + 1];
    }
    return pack8(y);
  }
  if (r.wide) {
    unpack8(k.other, g);
    const bool second = c >= r.half;
    const float2* const t = angles + (second ? c - r.half : c);
#pragma unroll
    for (int j = 0; j < 8; ++j) y[j] = second ? rotary_second(g[j], f[j], t[j]) : rotary_first(f[j], g[j], t[j]);
    return pack8(y);
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const int ch = c + j;
    y[j] = f[j];
    if (ch >= 2 * r.half) continue;
    const bool second = ch >= r.half;
    const int pair = second ? ch - r.half : ch;
    const float other = __half2float(head[second ? pair : pair + r.half]);
    y[j] = second ? rotary_second(other, f[j], angles[pair]) : rotary_first(f[j], other, angles[pair]);
  }
  return pack8(y);
}

// The pages' rows of K or V and a head, from the block blockIdx.x of those that the
// sequence's new tokens fall into, by steps of gridDim.x.
template <int D, bool IS_V>
__device__ __forceinline__ void append_pages(const AppendArgs& a, const Rotary& r, const KvSeq& q, uint4* stage,
                                             float2 (*angles)[256]) {
  constexpr int kOctets = D / 8;               // of channels
  constexpr int kStep = kThreads / kOctets;    // slots that the threads' octets cover at a time
  constexpr int kWaveSlots = 64 / kOctets;     // and a wave's
  constexpr int kPairs = D / 2, kFreqs = kPairs > 64 ? kPairs / 64 : 1;
  static_assert(kWaveSlots * kPairs == 256, "a wave's angles");
  const int b = blockIdx.z, tid = threadIdx.x;
  const int head = (int)blockIdx.y >> 1;
  const int octet = tid % kOctets, c = 8 * octet;
  const int lane = tid & 63, wave = tid >> 6;
  float2* const mine = angles[wave];
  // The frequencies of the lane's pairs, ahead of the table and the rows.
  double freq[kFreqs] = {};
  if constexpr (!IS_V) {
#pragma unroll
    for (int n = 0; n < kFreqs; ++n) {
      const int pair = (lane + 64 * n) % kPairs;
      if (pair < r.half) freq[n] = r.inv_freq[pair];
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
    uint8_t* const codes = a.pages[IS_V] + at * (kPage * D);
    const float had = fresh ? 0.0f : a.scales[IS_V][at];

    // The new tokens' rows into LDS, and their largest magnitude.  V's octets are
    // turned by the slot's eighth, for the reads by channels below: the 64 lanes
    // then read 32 dwords of as many banks.
    float top = 0.0f;
    const __half* const row0 = a.x[IS_V] + (int64_t)head * D;
    const int from = lo / kStep * kStep;
#pragma unroll 1
    for (int first = from; first < hi; first += kStep) {
      const int slot = first + tid / kOctets;
      const int64_t row = (int64_t)q.first_row + ((int64_t)(blk * kPage + slot) - q.start);
      const __half* const x = row0 + row * a.ld[IS_V];
      const bool is_new = slot >= lo && slot < hi;
      KeyOctet k{};
      if (is_new) k = key_octet(r, x, c, !IS_V);
      if constexpr (!IS_V) {
        // The angles of the wave's tokens.
#pragma unroll 2
        for (int n = 0; n < kWaveSlots * kPairs / 64; ++n) {
          const int at = 64 * n + lane, s = first + wave * kWaveSlots + at / kPairs;
          if (s >= lo && s < hi && at % kPairs < r.half)
            mine[at] = rotary_angle(blk * kPage + s, freq[n % kFreqs], r.scale);
        }
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
      }
      if (is_new) {
        if constexpr (!IS_V) k.v = rotate_octet(r, k, x, c, mine + lane / kOctets * kPairs);
        float f[8];
        unpack8(k.v, f);
#pragma unroll
        for (int j = 0; j < 8; ++j) top = fmaxf(top, fabsf(f[j]));
        stage[slot * kOctets + (IS_V ? octet ^ (slot >> 3) : octet)] = k.v;
      }
      if constexpr (!IS_V) {
        // The next angles wait for these reads.
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
      }
    }
    top = wave_max(top);
    if (lane == 0) mine->x = top;
    __syncthreads();   // and everyone has read the scale
#pragma unroll
    for (int i = 0; i < kWaves; ++i) top = fmaxf(top, angles[i][0].x);
    const float s = fmaxf(__uint_as_float((uint32_t)(scale_exp(top) + 127) << 23), had);
    const bool grew = !fresh && s > had;
    const float ratio = had / s, inv = 1.0f / s;   // exact for powers of two
    if (tid == 0) a.scales[IS_V][at] = s;

    if constexpr (!IS_V) {
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
      // Units: a channel and eight slots, of the eighths of the page that change.
      const __half* const staged = reinterpret_cast<const __half*>(stage);
      const int low = fresh || grew ? 0 : lo / 8, eighths = (fresh ? 8 : (hi + 7) / 8) - low;
      const int share = (0xFFFF + eighths) / eighths;   // u / eighths = u share / 2^16
#pragma unroll 1
      for (int u = tid; u < eighths * D; u += kThreads) {
        const int d = u * share >> 16, eighth = low + u - d * eighths, first = 8 * eighth;
        uint8_t* const dst = codes + d * kPage + first;
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
    __syncthreads();   // angles and stage are free again
  }
}

template <int D>
__global__ void __launch_bounds__(kThreads) rotary_append_kernel(AppendArgs a, RotaryQ rq) {
  // The page's rows, an octet of slot s at s * D / 8 + (octet ^ turn(s)).
  __shared__ uint4 stage[kPage * D / 8];
  // Of each wave: the angles of the tokens that its lanes have octets of (or of one
  // token), then its largest magnitude.
  __shared__ float2 angles[kWaves][256];
  const KvSeq q = kv_seq(a.cu, a.lengths, blockIdx.z, a.T);
  if ((int)blockIdx.y >= 2 * a.heads) {
    float2* const mine = angles[threadIdx.x >> 6];
    const int slice = (int)blockIdx.y - 2 * a.heads, slices = (int)gridDim.y - 2 * a.heads;
    if (rq.r.interleaved)
      rq.r.wide ? rotate_q<true, true>(rq, q, slice, slices, mine) : rotate_q<true, false>(rq, q, slice, slices, mine);
    else
      rq.r.wide ? rotate_q<false, true>(rq, q, slice, slices, mine) : rotate_q<false, false>(rq, q, slice, slices, mine);
    return;
  }
  if (q.count == 0 || q.length == 0) return;
  if (blockIdx.y & 1)
    append_pages<D, true>(a, rq.r, q, stage, angles);
  else
    append_pages<D, false>(a, rq.r, q, stage, angles);
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
  // A wave to each token and part, behind the pages' workgroups, whose chains of
  // loads are the longer ones (queries first: 46 us for 40, 4500 tokens).  More than
  // 64 angles a token are two rounds of a wave's lanes: up to four parts then share
  // them while 4096 waves are left (3 x 415 tokens of 64 heads of 256: 28 against 31.5
  // us; with 64 angles, 4500 tokens of 64 heads of 128, 39.7 against 35).
  const int64_t share = c.T * rq.parts / 4096;
  rq.run = rq.r.half <= 64 || share < 1 ? 1 : share < 4 ? (int)share : 4;
  rq.pieces = (rq.parts + rq.run - 1) / rq.run;
  const int64_t waves = (max_new < 64 ? max_new : 64) * rq.pieces;
  const int64_t slices = (waves + kWaves - 1) / kWaves;
  // Tiles of 64 tokens, and pages, that max_new tokens can touch; more loop.
  const int64_t tiles = (max_new + kPage - 2) / kPage + 1;
  const dim3 grid((unsigned)(tiles < 65535 ? tiles : 65535),
                  (unsigned)(2 * c.kv_heads + (slices < 1024 ? slices : 1024)), (unsigned)c.B);
  switch (c.head_dim) {
    case 64: launch<64>(a, rq, grid, stream); break;
    case 128: launch<128>(a, rq, grid, stream); break;
    case 256: launch<256>(a, rq, grid, stream); break;
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

}  // namespace dptq
