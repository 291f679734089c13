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
#include "internal.h"
#include "kv8_write.h"
#include "wave_device.h"

namespace dptq {
namespace {

constexpr int kThreads = 256;

template <int D>
__global__ void __launch_bounds__(kThreads) kv8_append_kernel(AppendArgs a) {
  constexpr int kOctets = D / 8;                       // of channels
  constexpr int kPer = kPage * kOctets / kThreads;     // tokens x octets of a thread
  constexpr int kRow = kPage + 4;                      // of the staged V codes, a channel a row
  __shared__ float part[kThreads / 64];
  __shared__ __align__(8) uint8_t stage[D * kRow];
  const int b = blockIdx.z, head = blockIdx.y >> 1;
  const bool is_v = blockIdx.y & 1;
  const KvSeq q = kv_seq(a.cu, a.lengths, b, a.T);
  if (q.count == 0 || q.length == 0) return;
  const int begin = max(q.start, 0);
  const int last_block = min((q.length - 1) / kPage, a.max_pages - 1);
  const int tid = threadIdx.x;
  // A thread's tokens of one octet of channels: for K every (64 / kPer)th, so
  // that a row's octets are stored by consecutive threads; for V consecutive
  // ones, which make one LDS store of a channel.
  const int octet = tid % kOctets, first_slot = tid / kOctets * (is_v ? kPer : 1);
  const int slot_step = is_v ? 1 : kPage / kPer;
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

}  // namespace

hipError_t launch_kv8_append(const Kv8Cache& c, const void* k, int64_t ld_k, const void* v, int64_t ld_v,
                             int64_t max_new, hipStream_t stream) {
  const AppendArgs a = append_args(c, k, ld_k, v, ld_v);
  // Pages that max_new tokens can touch; a sequence with more loops.
  int64_t blocks = (max_new + kPage - 2) / kPage + 1;
  blocks = blocks < c.max_pages ? blocks : c.max_pages;
  const dim3 grid((unsigned)(blocks < 65535 ? blocks : 65535), (unsigned)(2 * c.kv_heads), (unsigned)c.B);
  switch (c.head_dim) {
    case 64: kv8_append_kernel<64><<<grid, kThreads, 0, stream>>>(a); break;
    case 128: kv8_append_kernel<128><<<grid, kThreads, 0, stream>>>(a); break;
    case 256: kv8_append_kernel<256><<<grid, kThreads, 0, stream>>>(a); break;
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

}  // namespace dptq
