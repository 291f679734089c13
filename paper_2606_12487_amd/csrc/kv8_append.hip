// New keys and values into the 8-bit paged cache (layout: kv8_device.h).
//
// A workgroup takes one page that new tokens of a sequence fall into, one KV
// head, and K or V.  With a the largest |x| of the page's new tokens:
//
//   e = the smallest integer >= -32 with a <= 448 * 2^e
//   s = max(2^e, the page's scale so far)      (2^e where the page is new)
//   code = e4m3(x / s), and where s grew the older codes become
//   e4m3(code * s_old / s).
//
// Scales are powers of two, so a larger one costs the older codes nothing but
// what falls below e4m3's normal range: tokens that arrive one by one give
// nearly the codes of a prompt written at once.  448 / 2^e wastes less than a
// factor of two of a floating-point format's range, which e4m3 does not feel.
//
// A page that is new (its first slot is written now) has its other slots
// cleared.  2 bytes read and 1 written per element; bound by latency: the loads
// of offsets, table and rows in turn (the rows are loaded once the table's entry
// is known to be a page, though their addresses do not depend on it) and the
// reduction behind them.  A token for each of 64 sequences (8 heads of 128) takes
// 7.4 us, 4500 tokens of three prompts 10.1 us (2.6 TB/s), at three workgroups
// on a compute unit.
//
// With rotary positions (kv8_append_kernel<D, true>) the keys are rotated and
// rounded to fp16 first, and wait in LDS for the page's scale: a workgroup of K
// loads the other channel of each pair too (a second load of bytes that its
// neighbour loads) and computes its own angles.  Further workgroups rotate the
// queries, a token and a part of its heads to a wave.  The codes are those of
// rotary and kv8_append one after the other, bit for bit.  The queries' way is
// bound by bytes, and so by the loads in flight, which the kernel's registers
// limit: three workgroups on a compute unit (two at 256 channels).  4500 tokens
// of three prompts with 64 heads of queries take 40 us (4.2 TB/s; 60 us with the
// keys' loops unrolled, at two workgroups), a token for each of 64 sequences 10.2.
#include "internal.h"
#include "kv8_device.h"
#include "rotary_device.h"
#include "wave_device.h"

namespace dptq {
namespace {

constexpr int kThreads = 256;

struct AppendArgs {
  const __half* x[2];   // K, V rows
  int64_t ld[2];
  uint8_t* pages[2];
  float* scales[2];
  const int32_t *cu, *lengths, *table;
  int T, max_pages, num_pages, heads;
};

// The queries' side of a call with rotary positions.
struct RotaryQ {
  Rotary r;
  const __half* q;
  __half* out;
  int64_t ld, ld_out;
  int heads, parts;   // parts of 256 units
};
constexpr int kRotaryUnits = 4;   // of a lane

// Rotates the queries of tokens [64 x, 64 x + 64) of a sequence, and so on by
// gridDim.x; the workgroup is slice `slice` of `slices` of them.
template <bool INTER, bool WIDE>
__device__ __forceinline__ void rotate_q(const RotaryQ& a, const KvSeq& s, int slice, int slices, float2* angles) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  for (int64_t first = 64 * (int64_t)blockIdx.x; first < s.count; first += 64 * (int64_t)gridDim.x) {
    const int tokens = (int)min((int64_t)64, s.count - first);
    for (int i = slice * (kThreads / 64) + wave; i < tokens * a.parts; i += slices * (kThreads / 64)) {
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
    for (int j = 0; j < 8; ++j) g[j] = f[j ^ 1];
  } else if (r.wide) {
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
    if (ch >= 2 * r.half) continue;   // an octet that the pairs end in
    const bool second = r.interleaved ? ch & 1 : ch >= r.half;
    const float2 t = rotary_angle(p, freq[j], r.scale);
    y[j] = second ? rotary_second(g[j], f[j], t) : rotary_first(f[j], g[j], t);
  }
  return pack8(y);
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

// The keys of a page, rotated, into the cache: rounded to fp16 they wait in LDS
// (stage) for the page's scale.  Loops that are not unrolled keep the kernel's
// registers, which the workgroups of the queries have too, few.
template <int D>
__device__ __forceinline__ void rotary_page(const Rotary& r, const KvSeq& q, int blk, int lo, int hi, const __half* head,
                                            int64_t ld, uint8_t* codes, float* scale, float had, int octet,
                                            int first_slot, int slot_step, const double (&freq)[8], uint4* stage,
                                            float* part) {
  constexpr int kPer = kPage * (D / 8) / kThreads;
  const int tid = threadIdx.x, c = 8 * octet;
  const bool fresh = lo == 0;
  float top = 0.0f;
#pragma unroll 1
  for (int i = 0; i < kPer; ++i) {
    const int slot = first_slot + i * slot_step;
    if (slot < lo || slot >= hi) continue;
    const int p = blk * kPage + slot;
    const __half* const row = head + ((int64_t)q.first_row + ((int64_t)p - q.start)) * ld;
    const uint4 v = rotate_octet(r, *reinterpret_cast<const uint4*>(row + c), row, c, p, freq);
    float f[8];
    unpack8(v, f);
#pragma unroll
    for (int j = 0; j < 8; ++j) top = fmaxf(top, fabsf(f[j]));
    stage[i * kThreads + tid] = v;
  }
  top = wave_max(top);
  if ((tid & 63) == 0) part[tid / 64] = top;
  __syncthreads();   // and everyone has read the scale
#pragma unroll
  for (int i = 0; i < kThreads / 64; ++i) top = fmaxf(top, part[i]);
  const float s = fmaxf(__uint_as_float((uint32_t)(scale_exp(top) + 127) << 23), had);
  const bool grew = !fresh && s > had;
  const float ratio = had / s, inv = 1.0f / s;   // exact for powers of two
  if (tid == 0) *scale = s;
#pragma unroll 1
  for (int i = 0; i < kPer; ++i) {
    const int slot = first_slot + i * slot_step;
    uint2* const dst = reinterpret_cast<uint2*>(codes + slot * D + c);
    if (slot >= lo && slot < hi) {
      float f[8];
      unpack8(stage[i * kThreads + tid], f);
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
  __syncthreads();   // part is free again
}

template <int D, bool ROTARY>
__global__ void __launch_bounds__(kThreads, !ROTARY ? 1 : D == 256 ? 2 : 3) kv8_append_kernel(AppendArgs a, RotaryQ rq) {
  constexpr int kOctets = D / 8;                       // of channels
  constexpr int kPer = kPage * kOctets / kThreads;     // tokens x octets of a thread
  constexpr int kRow = kPage + 4;                      // of the staged V codes, a channel a row
  __shared__ float part[kThreads / 64];
  // The staged V codes, or the page's rotated keys, or a token's angles in each wave.
  __shared__ __align__(16) uint8_t stage[ROTARY ? kPage * D * 2 : D * kRow];
  const int b = blockIdx.z, head = (int)blockIdx.y >> 1;
  const bool is_v = blockIdx.y & 1;
  const KvSeq q = kv_seq(a.cu, a.lengths, b, a.T);
  if constexpr (ROTARY) {
    if ((int)blockIdx.y >= 2 * a.heads) {
      float2* const mine = reinterpret_cast<float2*>(stage) + (threadIdx.x >> 6) * (D / 2);
      const int slice = (int)blockIdx.y - 2 * a.heads, slices = (int)gridDim.y - 2 * a.heads;
      if (rq.r.interleaved)
        rq.r.wide ? rotate_q<true, true>(rq, q, slice, slices, mine) : rotate_q<true, false>(rq, q, slice, slices, mine);
      else
        rq.r.wide ? rotate_q<false, true>(rq, q, slice, slices, mine)
                  : rotate_q<false, false>(rq, q, slice, slices, mine);
      return;
    }
  }
  if (q.count == 0 || q.length == 0) return;
  const int begin = max(q.start, 0);
  const int last_block = min((q.length - 1) / kPage, a.max_pages - 1);
  const int tid = threadIdx.x;
  // A thread's tokens of one octet of channels: for K every (64 / kPer)th, so
  // that a row's octets are stored by consecutive threads; for V consecutive
  // ones, which make one LDS store of a channel.
  const int octet = tid % kOctets, first_slot = tid / kOctets * (is_v ? kPer : 1);
  const int slot_step = is_v ? 1 : kPage / kPer;
  // The frequencies of the octet's channels, ahead of the table and the rows.
  double freq[8] = {};
  if constexpr (ROTARY) {
    if (!is_v) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int ch = 8 * octet + j;
        const int pair = rq.r.interleaved ? ch >> 1 : ch >= rq.r.half ? ch - rq.r.half : ch;
        if (ch < 2 * rq.r.half) freq[j] = rq.r.inv_freq[pair];
      }
    }
  }
  for (int blk = begin / kPage + blockIdx.x; blk <= last_block; blk += gridDim.x) {
    const int page = a.table[(int64_t)b * a.max_pages + blk];
    if ((uint32_t)page >= (uint32_t)a.num_pages) continue;
    const int lo = max(begin - blk * kPage, 0);                    // new slots [lo, hi)
    const int hi = min(q.length - blk * kPage, kPage);
    const bool fresh = lo == 0;
    const int64_t at = (int64_t)page * a.heads + head;
    uint8_t* const codes = a.pages[is_v] + at * (kPage * D);
    const __half* const rows = a.x[is_v] + (int64_t)head * D + 8 * octet;
    const float had = fresh ? 0.0f : a.scales[is_v][at];

    if constexpr (ROTARY) {
      if (!is_v) {
        rotary_page<D>(rq.r, q, blk, lo, hi, rows - 8 * octet, a.ld[0], codes, a.scales[0] + at, had, octet, first_slot,
                       slot_step, freq, reinterpret_cast<uint4*>(stage), part);
        continue;
      }
    }

    // The new tokens' values and their largest magnitude.
    uint4 v[kPer];
    float top = 0.0f;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int slot = first_slot + i * slot_step;
      v[i] = make_uint4(0, 0, 0, 0);
      if (slot >= lo && slot < hi) {
        const int64_t t = (int64_t)q.first_row + ((int64_t)blk * kPage + slot - q.start);
        v[i] = *reinterpret_cast<const uint4*>(rows + t * a.ld[is_v]);
      }
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const uint32_t w[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const __half2 h = *reinterpret_cast<const __half2*>(&w[j]);
        top = fmaxf(top, fmaxf(fabsf(__low2float(h)), fabsf(__high2float(h))));
      }
    }
    top = wave_max(top);
    if ((tid & 63) == 0) part[tid / 64] = top;
    __syncthreads();   // and everyone has read the scale
#pragma unroll
    for (int i = 0; i < kThreads / 64; ++i) top = fmaxf(top, part[i]);
    const float need = __uint_as_float((uint32_t)(scale_exp(top) + 127) << 23);
    const float s = fmaxf(need, had);
    const bool grew = !fresh && s > had;
    const float ratio = had / s, inv = 1.0f / s;   // exact for powers of two
    if (tid == 0) a.scales[is_v][at] = s;

    float f[kPer][8];
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const uint32_t w[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const __half2 h = *reinterpret_cast<const __half2*>(&w[j]);
        f[i][2 * j] = __low2float(h) * inv;
        f[i][2 * j + 1] = __high2float(h) * inv;
      }
    }
    if (!is_v) {
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        const int slot = first_slot + i * slot_step;
        uint2* const dst = reinterpret_cast<uint2*>(codes + slot * D + 8 * octet);
        if ((slot >= lo && slot < hi) || (fresh && slot >= hi)) {
          *dst = make_uint2(to_e4m3<true>(f[i][2], f[i][3], to_e4m3<false>(f[i][0], f[i][1], 0)),
                            to_e4m3<true>(f[i][6], f[i][7], to_e4m3<false>(f[i][4], f[i][5], 0)));
        } else if (slot < lo && grew) {
          const uint2 o = *dst;
          *dst = make_uint2(rescale4(o.x, ratio), rescale4(o.y, ratio));
        }
      }
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        uint8_t* const to = stage + (8 * octet + j) * kRow + first_slot;
        if constexpr (kPer == 2) {
          *reinterpret_cast<uint16_t*>(to) = (uint16_t)to_e4m3<false>(f[0][j], f[1][j], 0);
        } else {
#pragma unroll
          for (int i = 0; i < kPer; i += 4)
            *reinterpret_cast<uint32_t*>(to + i) =
                to_e4m3<true>(f[i + 2][j], f[i + 3][j], to_e4m3<false>(f[i][j], f[i + 1][j], 0));
        }
      }
      __syncthreads();
      // Unit u: channel u / 8, slots 8 (u % 8) and up.
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        const int u = tid + i * kThreads, d = u / 8, first = 8 * (u % 8);
        const uint32_t* const from = reinterpret_cast<const uint32_t*>(stage + d * kRow + first);
        uint8_t* const dst = codes + d * kPage + first;
        const uint2 n = make_uint2(from[0], from[1]);
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

AppendArgs append_args(const Kv8Cache& c, const void* k, int64_t ld_k, const void* v, int64_t ld_v) {
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

template <bool ROTARY>
hipError_t launch(const AppendArgs& a, const RotaryQ& rq, int head_dim, dim3 grid, hipStream_t stream) {
  switch (head_dim) {
    case 64: kv8_append_kernel<64, ROTARY><<<grid, kThreads, 0, stream>>>(a, rq); break;
    case 128: kv8_append_kernel<128, ROTARY><<<grid, kThreads, 0, stream>>>(a, rq); break;
    case 256: kv8_append_kernel<256, ROTARY><<<grid, kThreads, 0, stream>>>(a, rq); break;
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

// Workgroups along a sequence's new tokens, for what `most` tiles of 64 hold.
unsigned tiles(int64_t most) { return (unsigned)(most < 1 ? 1 : most < 65535 ? most : 65535); }

}  // namespace

hipError_t launch_kv8_append(const Kv8Cache& c, const void* k, int64_t ld_k, const void* v, int64_t ld_v,
                             int64_t max_new, hipStream_t stream) {
  // Pages that max_new tokens can touch; a sequence with more loops.
  const int64_t blocks = (max_new + kPage - 2) / kPage + 1;
  const dim3 grid(tiles(blocks < c.max_pages ? blocks : c.max_pages), (unsigned)(2 * c.kv_heads), (unsigned)c.B);
  return launch<false>(append_args(c, k, ld_k, v, ld_v), RotaryQ{}, c.head_dim, grid, stream);
}

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
  const int64_t slices = (waves + kThreads / 64 - 1) / (kThreads / 64);
  const dim3 grid(tiles((max_new + kPage - 2) / kPage + 1), (unsigned)(2 * c.kv_heads + (slices < 1024 ? slices : 1024)),
                  (unsigned)c.B);
  return launch<true>(a, rq, c.head_dim, grid, stream);
}

}  // namespace dptq
