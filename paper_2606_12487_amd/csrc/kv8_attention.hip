// Attention of new queries over the 8-bit paged cache (layout: kv8_device.h).
//
// Query i of a sequence of length n with c new queries stands at position
// p = n - c + i and sees positions j <= p, with a window W only those with
// j > p - W or j < sinks.  For query head a of KV head h:
//
//   S_j = scale * s_k[page(j), h] * (q . kc_j),   P = softmax(S over visible j)
//   out = sum_j P_j s_v[page(j), h] vc_j,         lse = log sum_j exp(S_j)
//
// (kc, vc: the e4m3 codes.)  A row that sees nothing gives 0 and -inf.
//
// One pass over the keys with the softmax's sum l in base 2, relative to a
// reference m that follows the running maximum (below).  fp32 throughout except
// P, which is rounded to fp16 as an operand of the second product: half to even,
// a relative error up to 2^-11 of a weight, absolute 2^-25 below 2^-14, where the
// row's largest weight is 1 or more.  That adds up to a quarter to the error of
// the outputs' own rounding to fp16 (2.6e-4 against 2.1e-4 of their size).
// Codes are exact in fp16, queries are taken as they are, and the scales are
// applied in fp32: k's to the scores, v's as its ratio to the unit in which the
// output accumulates.
//
// Both products run on the matrix cores transposed: S^T = K Q^T has the page's
// tokens as rows and the queries as columns, O^T = V^T P^T the channels as
// rows.  The rows of the K operand are taken in an order that leaves each lane
// with the scores of 16 consecutive tokens of one query, which is exactly what
// the second product wants of P from that lane: P never leaves the registers.
#include "kv8_attn.h"

namespace dptq {
namespace {

// 16 bytes that no other workgroup reads: past the caches' retention (2 % less
// time on 64 sequences of up to 8192 tokens, 10 % with 32 key heads).
__device__ __forceinline__ uint4 stream16(const uint8_t* p) {
  typedef uint32_t uint4v __attribute__((ext_vector_type(4)));
  const uint4v x = __builtin_nontemporal_load(reinterpret_cast<const uint4v*>(p));
  return make_uint4(x[0], x[1], x[2], x[3]);
}

// 16 rows (queries of one KV head of one sequence; row r is query token
// r / group, head r % group of the group) by one part of the visible pages.
// Each of the four waves takes every fourth page of the part, straight from
// memory into the registers that feed the matrix cores: K of the next page is
// loaded behind the scores, V behind the second product.
//
// The softmax keeps a reference m instead of the running maximum: weights are
// 2^(s - m), and m moves (with the sums and O rescaled) only where a score
// passes m + 10, then to 4 below it.  A page's v scale goes into the exponent
// as its ratio to the unit U of O, 2^-4 to 2^4; another unit is taken, with O
// rescaled, where the ratio leaves that range.  Weights stay below 2^15, within
// fp16, and are never below their exact size relative to the row's largest.
//
// Bound by the bytes of the cache: 64 sequences of up to 8192 tokens (64 heads
// on 8, head size 128) take 141 us, 4.9 TB/s; two of up to 131072 take 86 us,
// 5.3 TB/s; 16 with 32 key heads behind a window of 4096 take 90 us, 6.0 TB/s
// (a plain read stream reaches 7.1).
template <int D>
__global__ void __launch_bounds__(256, D == 64 ? 4 : D == 128 ? 2 : 1) kv8_decode_kernel(AttnArgs a) {
  constexpr int kC = D / 64;     // 64-channel parts of a row
  constexpr int kT = D / 16;     // 16-channel tiles of the output
  constexpr int kSlots = D == 256 ? 2 : 4;   // waves whose outputs stand in LDS at once
  __shared__ float sum_o[kSlots][16 * D];
  __shared__ float2 wave_ml[4][16];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int col = lane & 15, quad = lane >> 4;
  const int head = (int)blockIdx.x, b = (int)blockIdx.z / a.splits, part = (int)blockIdx.z % a.splits;
  const KvSeq seq = kv_seq(a.cu, a.lengths, b, a.T);
  const int rows = seq.count * a.group;   // T * heads < 2^30
  const int32_t* const table = a.table + (int64_t)b * a.max_pages;
  const float sign = a.scale_log2 < 0.0f ? -1.0f : 1.0f;

  for (int row0 = (int)blockIdx.y * 16; row0 < rows; row0 += (int)gridDim.y * 16) {
    const int row = min(row0 + col, rows - 1);    // lanes past the end repeat the last row
    const int token = row / a.group, g = row % a.group;
    const int pos = seq.start + token;
    const int pmin = seq.start + row0 / a.group;
    const int pmax = seq.start + min(row0 + 15, rows - 1) / a.group;
    const Visible vis = visible_pages(pmin, pmax, a.window, a.sinks, a.max_pages);
    const int begin = min(part * a.chunk, vis.total);
    const int end = part == a.splits - 1 ? vis.total : min(begin + a.chunk, vis.total);

    // Queries: chunk (C, e) of 32 channels gives lane (col, quad) the channels
    // 64 C + 16 quad + 8 e and up, as K's 16-byte loads hold them.
    half8 qf[kC][2];
    const __half* const qrow = a.q + (int64_t)(seq.first_row + token) * a.ld_q + (int64_t)(head * a.group + g) * D;
#pragma unroll
    for (int C = 0; C < kC; ++C)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        qf[C][e] = *reinterpret_cast<const half8*>(qrow + 64 * C + 16 * quad + 8 * e);
        qf[C][e] *= (_Float16)sign;
      }

    float4v o[kT];
#pragma unroll
    for (int t = 0; t < kT; ++t) o[t] = float4v{0, 0, 0, 0};
    float m = -INFINITY, l = 0.0f, unit = 0.0f;   // unit 0: none yet

    // S^T: row x of tile t4 is token 16 (x / 4) + 4 t4 + x % 4, so that lane
    // (col, quad) ends with tokens 16 quad + 4 t4 + i.
    uint4 kc[4][kC], vc[kT];
    const uint32_t k_at = (uint32_t)((16 * (col >> 2) + (col & 3)) * D + 16 * quad);
    const uint32_t v_at = (uint32_t)(col * kPage + 16 * quad);
    // A page that is not there: page 0 is read, and all of it is masked.
    const auto there = [&](int page) { return (uint32_t)page < (uint32_t)a.num_pages; };
    const auto which = [&](int page) { return (int64_t)(there(page) ? page : 0) * a.kv_heads + head; };
    const auto load_k = [&](int64_t at) {
#pragma unroll
      for (int t4 = 0; t4 < 4; ++t4)
#pragma unroll
        for (int C = 0; C < kC; ++C)
          kc[t4][C] = stream16(a.k_pages + at * (kPage * D) + k_at + 4 * t4 * D + 64 * C);
    };
    const auto load_v = [&](int64_t at) {
#pragma unroll
      for (int t = 0; t < kT; ++t)
        vc[t] = stream16(a.v_pages + at * (kPage * D) + v_at + 16 * t * kPage);
    };

    int i = begin + wave;
    if (i < end) {
      int page = table[vis.page(i)];
      int page1 = i + 4 < end ? table[vis.page(i + 4)] : -1;
      load_k(which(page));
      load_v(which(page));
      float ks = a.k_scales[which(page)], vs = a.v_scales[which(page)];
      for (; i < end; i += 4) {
        const bool more = i + 4 < end;
        const int page2 = i + 8 < end ? table[vis.page(i + 8)] : -1;
        float s[16];
#pragma unroll
        for (int t4 = 0; t4 < 4; ++t4) {
          float4v acc = {0, 0, 0, 0};
#pragma unroll
          for (int C = 0; C < kC; ++C) {
            acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(codes8(kc[t4][C].x, kc[t4][C].y), qf[C][0], acc, 0, 0, 0);
            acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(codes8(kc[t4][C].z, kc[t4][C].w), qf[C][1], acc, 0, 0, 0);
          }
#pragma unroll
          for (int e = 0; e < 4; ++e) s[4 * t4 + e] = acc[e];
        }
        const float c = fmaxf(fabsf(a.scale_log2) * ks, 1e-37f);   // > 0 also where the scale is 0: -inf stays -inf
        const float v_scale = vs;
        if (more) {
          load_k(which(page1));
          ks = a.k_scales[which(page1)];
          vs = a.v_scales[which(page1)];
        }
        const bool here = there(page);
        const int j0 = vis.page(i) * kPage;
        if (!here || !page_whole(j0, pmin, pmax, a.window, a.sinks)) {
#pragma unroll
          for (int e = 0; e < 16; ++e)
            s[e] = here && sees(pos, j0 + 16 * quad + e, a.window, a.sinks) ? s[e] : -INFINITY;
        }
        float top = s[0];
#pragma unroll
        for (int e = 1; e < 16; ++e) top = fmaxf(top, s[e]);
        top *= c;
        const float ratio = unit > 0.0f ? v_scale / unit : 0.0f;
        const bool other_unit = !(ratio >= 0.0625f && ratio <= 16.0f) && here;
        if (__any(top > m + 10.0f) || other_unit) {
          // The four lanes of a row move its reference alike.
          float row_top = fmaxf(top, __shfl_xor(top, 16));
          row_top = fmaxf(row_top, __shfl_xor(row_top, 32));
          const float m_new = row_top > m + 10.0f ? row_top - 4.0f : m;
          const float alpha = m == -INFINITY ? 0.0f : exp2_hw(m - m_new);
          const float fix = alpha * (other_unit && unit > 0.0f ? unit / v_scale : 1.0f);
          if (other_unit) unit = v_scale;
          m = m_new;
          l *= alpha;
#pragma unroll
          for (int t = 0; t < kT; ++t) o[t] *= fix;
        }
        // Weights with the v scale in them; their sum without it.
        const float base = m == -INFINITY ? 0.0f : m;
        const float by = here ? v_scale / unit : 1.0f;
        const float shift = __builtin_amdgcn_logf(by) - base;
        half8 p[2];
        float sum = 0.0f;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const float x = exp2_hw(fmaf(s[e], c, shift));
          sum += x;
          p[e / 8][e % 8] = (_Float16)x;
        }
        l = fmaf(sum, 1.0f / by, l);
        // O^T: lane (col, quad) gives channel 16 t + col of tokens 16 quad and
        // up.  Slots past the sequence's end, and page 0 in place of one that is
        // not there, may hold anything: no NaN of theirs may meet the zero weight.
        if (!here || j0 + kPage > seq.length) {
          const int held = here ? seq.length - j0 - 16 * quad : 0;   // valid slots of this lane's 16
#pragma unroll
          for (int t = 0; t < kT; ++t) {
            vc[t].x &= held_mask(held, 0);
            vc[t].y &= held_mask(held, 4);
            vc[t].z &= held_mask(held, 8);
            vc[t].w &= held_mask(held, 12);
          }
        }
#pragma unroll
        for (int t = 0; t < kT; ++t) {
          o[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(codes8(vc[t].x, vc[t].y), p[0], o[t], 0, 0, 0);
          o[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(codes8(vc[t].z, vc[t].w), p[1], o[t], 0, 0, 0);
        }
        if (more) load_v(which(page1));
        page = page1;
        page1 = page2;
      }
    }
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);

    // Join the waves.
    if (quad == 0) wave_ml[wave][col] = make_float2(m, l);
    __syncthreads();
    float M = -INFINITY, L = 0.0f;
#pragma unroll
    for (int w = 0; w < 4; ++w) M = fmaxf(M, wave_ml[w][col].x);
    const float ref = M == -INFINITY ? 0.0f : M;
#pragma unroll
    for (int w = 0; w < 4; ++w) L += wave_ml[w][col].y * exp2_hw(wave_ml[w][col].x - ref);
    const float mine = exp2_hw(m - ref) * unit;
#pragma unroll
    for (int first = 0; first < 4; first += kSlots) {
      if (wave >= first && wave < first + kSlots) {
#pragma unroll
        for (int t = 0; t < kT; ++t) {
          float4v* const dst = reinterpret_cast<float4v*>(sum_o[wave % kSlots] + col * D + 16 * t + 4 * quad);
          *dst = first == 0 ? o[t] * mine : *dst + o[t] * mine;
        }
      }
      __syncthreads();
    }
    if (threadIdx.x < 16) wave_ml[0][threadIdx.x] = make_float2(M, L);   // lanes 0..15 hold rows 0..15
    __syncthreads();
    for (int e = threadIdx.x; e < 16 * D; e += 256) {
      const int r = row0 + e / D;
      if (r >= rows) break;
      const int d = e % D;
      const float2 ml = wave_ml[0][e / D];
      float x = 0.0f;
#pragma unroll
      for (int w = 0; w < kSlots; ++w) x += sum_o[w][e];
      const int64_t to = ((int64_t)seq.first_row + r / a.group) * a.heads + head * a.group + r % a.group;
      if (a.splits == 1) {
        a.out[to * D + d] = __float2half_rn(ml.y > 0.0f ? x / ml.y : ml.y);
        if (d == 0) a.lse[to] = ml.x * kLn2 + logf(ml.y);
      } else {
        const int64_t at = (int64_t)part * a.T * a.heads + to;
        if (begin < end) a.part_o[at * D + d] = x;   // parts without pages come last
        if (d == 0) a.part_ml[at] = ml;
      }
    }
    __syncthreads();
  }
}

// Joins the parts of one row, a wave a row: few parts.
constexpr int kFewSplits = 8;
template <int D>
__global__ void __launch_bounds__(256) kv8_combine_few_kernel(AttnArgs a) {
  constexpr int kV = D / 64;
  const int64_t n = (int64_t)a.T * a.heads;
  const int lane = threadIdx.x & 63;
  for (int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); row < n; row += (int64_t)gridDim.x * 4) {
    float2 ml[kFewSplits];
    float M = -INFINITY, L = 0.0f, o[kV] = {};
#pragma unroll
    for (int s = 0; s < kFewSplits; ++s) {
      ml[s] = s < a.splits ? a.part_ml[s * n + row] : make_float2(-INFINITY, 0.0f);
      M = fmaxf(M, ml[s].x);
    }
    const float ref = M == -INFINITY ? 0.0f : M;
#pragma unroll
    for (int s = 0; s < kFewSplits; ++s) {
      if (ml[s].y == 0.0f) continue;   // it saw nothing
      const float f = exp2_hw(ml[s].x - ref);
      L += f * ml[s].y;
#pragma unroll
      for (int i = 0; i < kV; ++i) o[i] += f * a.part_o[(s * n + row) * D + 64 * i + lane];
    }
#pragma unroll
    for (int i = 0; i < kV; ++i) a.out[row * D + 64 * i + lane] = __float2half_rn(L > 0.0f ? o[i] / L : L);
    if (lane == 0) a.lse[row] = M * kLn2 + logf(L);
  }
}

// The same, a workgroup a row, each wave every fourth part.
template <int D>
__global__ void __launch_bounds__(256) kv8_combine_kernel(AttnArgs a) {
  constexpr int kV = D / 64;
  __shared__ float factor[kMaxSplits];
  __shared__ float wave_max[4], wave_sum[4];
  __shared__ int wave_used[4];
  __shared__ float part[4][D];
  const int64_t n = (int64_t)a.T * a.heads;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int64_t row = blockIdx.x; row < n; row += gridDim.x) {
    float M = -INFINITY;
    int used = 0;   // parts up to the last that saw anything
    float2 ml[kMaxSplits / 256];
#pragma unroll
    for (int i = 0; i < kMaxSplits / 256; ++i) {
      const int s = threadIdx.x + 256 * i;
      ml[i] = s < a.splits ? a.part_ml[s * n + row] : make_float2(-INFINITY, 0.0f);
      M = fmaxf(M, ml[i].x);
      if (ml[i].y != 0.0f) used = s + 1;
    }
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) {
      M = fmaxf(M, __shfl_xor(M, off));
      used = max(used, __shfl_xor(used, off));
    }
    if (lane == 0) wave_max[wave] = M, wave_used[wave] = used;
    __syncthreads();
    used = max(max(wave_used[0], wave_used[1]), max(wave_used[2], wave_used[3]));
    M = fmaxf(fmaxf(wave_max[0], wave_max[1]), fmaxf(wave_max[2], wave_max[3]));
    const float ref = M == -INFINITY ? 0.0f : M;
    float L = 0.0f;
#pragma unroll
    for (int i = 0; i < kMaxSplits / 256; ++i) {
      const int s = threadIdx.x + 256 * i;
      const float f = exp2_hw(ml[i].x - ref);
      if (s < a.splits) factor[s] = f;
      L += f * ml[i].y;
    }
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) L += __shfl_xor(L, off);
    if (lane == 0) wave_sum[wave] = L;
    __syncthreads();
    L = (wave_sum[0] + wave_sum[1]) + (wave_sum[2] + wave_sum[3]);
    float o[kV] = {};
#pragma unroll 4
    for (int s = wave; s < used; s += 4) {
      const float* const src = a.part_o + (s * n + row) * D + lane;
      const float f = factor[s];
#pragma unroll
      for (int i = 0; i < kV; ++i) o[i] += f * src[64 * i];
    }
#pragma unroll
    for (int i = 0; i < kV; ++i) part[wave][64 * i + lane] = o[i];
    __syncthreads();
    for (int d = threadIdx.x; d < D; d += 256) {
      const float x = (part[0][d] + part[1][d]) + (part[2][d] + part[3][d]);
      a.out[row * D + d] = __float2half_rn(L > 0.0f ? x / L : L);
    }
    if (threadIdx.x == 0) a.lse[row] = M * kLn2 + logf(L);
    __syncthreads();
  }
}

// How a call is laid out: rows of a tile (16: the decode kernel), the pages of
// a part of what a tile sees, and the parts (the last one takes what is left).
struct Layout {
  int rows, chunk, splits;
};

Layout choose_layout(const Kv8Attention& c) {
  const int64_t group = c.heads / c.cache.kv_heads, heads = c.cache.B * c.cache.kv_heads, cus = device_cus();
  const auto tiles = [&](int64_t rows) { return (c.max_q * group + rows - 1) / rows * heads; };
  // The rows of a sequence that fit one tile of 16 go there (32 rows in two of
  // them take 42 us against 33 in one of 64: 16 sequences of 4096 tokens, 4
  // queries, 64 / 8 heads).  More go to tiles of 128, or of 64 while those are
  // fewer than two on a compute unit (256 tiles of 128 behind a window of 1024:
  // 29 us against 25 in 512 of 64).
  const int rows = c.max_q * group <= 16 ? 16 : tiles(128) >= 2 * cus ? 128 : 64;
  // What a tile sees: behind a window, that of its tokens, the sinks, and parts of pages at three ends.
  const int64_t seen = c.window > 0 ? c.window + (int64_t)c.sinks + rows / group + 1 + 3 * kPage : c.max_len;
  const int64_t pages = ((seen < c.max_len ? seen : c.max_len) + kPage - 1) / kPage;
  // Parts: for decode one round of the workgroups that a compute unit holds, 4,
  // 2 or 1 by the head size (at 128 two: 3, 4 and 8 took 1 to 15 % longer on the
  // large batches; at 256 one: 34 us against 42 for 65536 tokens), of four pages
  // (one a wave) or more, and none of what has up to eight pages (the second launch
  // costs more: 500 tokens 9.1 us against 10.7, while 777 take 11.4 against
  // 10.6); for prompts, whose partial outputs are large, only while there are
  // fewer tiles than compute units.
  const int64_t fill = rows == 16 ? 256 / c.cache.head_dim * cus : cus;
  int64_t chunk = (tiles(rows) * pages + fill - 1) / fill;
  chunk = (chunk + 3) / 4 * 4;
  const int64_t least = pages <= 8 ? 8 : 4;
  if (chunk < least) chunk = least;
  if (chunk * kMaxSplits < pages) chunk = (pages + kMaxSplits - 1) / kMaxSplits;
  const int64_t splits = pages < 1 ? 1 : (pages + chunk - 1) / chunk;
  return Layout{rows, (int)(chunk < 1 << 30 ? chunk : 1 << 30), (int)splits};
}

template <int D>
hipError_t launch(const AttnArgs& a, const Kv8Attention& c, int rows, hipStream_t stream) {
  hipError_t e;
  if (rows > 16) {
    e = launch_kv8_prompt(a, D, rows, c.cache.B, c.max_q, stream);
  } else {
    const int64_t tiles = (c.max_q * a.group + 15) / 16;
    // (There is more than one part only where there are few sequences: z fits.)
    const dim3 grid((unsigned)a.kv_heads, (unsigned)(tiles < 65535 ? tiles : 65535),
                    (unsigned)(c.cache.B * a.splits));
    kv8_decode_kernel<D><<<grid, 256, 0, stream>>>(a);
    e = hipGetLastError();
  }
  if (e != hipSuccess || a.splits == 1) return e;
  const int64_t out_rows = (int64_t)a.T * a.heads;
  const int64_t groups = a.splits <= kFewSplits ? (out_rows + 3) / 4 : out_rows;
  const unsigned grid = (unsigned)(groups < 65536 ? groups : 65536);
  if (a.splits <= kFewSplits) kv8_combine_few_kernel<D><<<grid, 256, 0, stream>>>(a);
  else kv8_combine_kernel<D><<<grid, 256, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace

int64_t kv8_attention_workspace(const Kv8Attention& c) {
  const int splits = choose_layout(c).splits;
  return splits == 1 ? 0 : (int64_t)splits * c.cache.T * c.heads * (c.cache.head_dim * 4 + 8);
}

hipError_t launch_kv8_attention(const Kv8Attention& c, hipStream_t stream) {
  AttnArgs a{};
  a.q = static_cast<const __half*>(c.q);
  a.ld_q = c.ld_q;
  a.k_pages = c.cache.k_pages;
  a.v_pages = c.cache.v_pages;
  a.k_scales = c.cache.k_scales;
  a.v_scales = c.cache.v_scales;
  a.cu = c.cache.cu;
  a.lengths = c.cache.lengths;
  a.table = c.cache.table;
  a.T = (int)c.cache.T;
  a.max_pages = c.cache.num_pages > 0 ? (int)c.cache.max_pages : 0;   // no pages: nothing is seen
  a.num_pages = (int)c.cache.num_pages;
  a.heads = c.heads;
  a.kv_heads = c.cache.kv_heads;
  a.group = c.heads / c.cache.kv_heads;
  a.scale_log2 = c.scale * kLog2e;
  a.window = c.window;
  a.sinks = c.sinks;
  const Layout layout = choose_layout(c);
  a.chunk = layout.chunk;
  a.splits = layout.splits;
  a.out = static_cast<__half*>(c.out);
  a.lse = c.lse;
  a.part_o = static_cast<float*>(c.workspace);
  a.part_ml = reinterpret_cast<float2*>(a.part_o + (int64_t)a.splits * a.T * a.heads * c.cache.head_dim);
  switch (c.cache.head_dim) {
    case 64: return launch<64>(a, c, layout.rows, stream);
    case 128: return launch<128>(a, c, layout.rows, stream);
    case 256: return launch<256>(a, c, layout.rows, stream);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace dptq
