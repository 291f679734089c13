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
// One pass over the keys with the running maximum m and sum l of the softmax
// in base 2, fp32 throughout except P, which is rounded to fp16 (half to even,
// relative error 2^-12 of a weight in (0, 1], absolute 2^-25 below 2^-14) as an
// operand of the second product.  Codes are exact in fp16, queries are taken
// as they are, and the scales are applied to fp32 sums: k's to the scores, v's
// by keeping the output accumulators in units of the current page's v scale.
//
// Both products run on the matrix cores transposed: S^T = K Q^T has the page's
// tokens as rows and the queries as columns, O^T = V^T P^T the channels as
// rows.  The rows of the K operand are taken in an order that leaves each lane
// with the scores of 16 consecutive tokens of one query, which is exactly what
// the second product wants of P from that lane: P never leaves the registers.
#include "kv8_attn.h"

namespace dptq {
namespace {

// 16 rows (queries of one KV head of one sequence; row r is query token
// r / group, head r % group of the group) by one split of the visible pages.
// Each of the four waves takes every fourth page of the split.
template <int D>
__global__ void __launch_bounds__(256) kv8_decode_kernel(AttnArgs a) {
  constexpr int kC = D / 64;     // 64-channel parts of a row
  constexpr int kT = D / 16;     // 16-channel tiles of the output
  __shared__ float sum_o[16 * D];
  __shared__ float2 wave_ml[4][16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int col = lane & 15, quad = lane >> 4;
  const int head = (int)blockIdx.x % a.kv_heads, b = (int)blockIdx.x / a.kv_heads;
  const KvSeq seq = kv_seq(a.cu, a.lengths, b, a.T);
  const int rows = seq.count * a.group;   // T * heads < 2^30

  for (int row0 = (int)blockIdx.y * 16; row0 < rows; row0 += (int)gridDim.y * 16) {
    const int row = min(row0 + col, rows - 1);    // lanes past the end repeat the last row
    const int token = row / a.group, g = row % a.group;
    const int pos = seq.start + token;
    const int pmin = seq.start + row0 / a.group;
    const int pmax = seq.start + min(row0 + 15, rows - 1) / a.group;
    const Visible vis = visible_pages(pmin, pmax, a.window, a.sinks, a.max_pages);
    const int begin = (int)((int64_t)vis.total * blockIdx.z / a.splits);
    const int end = (int)((int64_t)vis.total * (blockIdx.z + 1) / a.splits);

    // Queries: chunk (C, e) of 32 channels gives lane (col, quad) the channels
    // 64 C + 16 quad + 8 e and up, as K's 16-byte loads hold them.
    half8 qf[kC][2];
    const __half* const qrow = a.q + (int64_t)(seq.first_row + token) * a.ld_q + (int64_t)(head * a.group + g) * D;
#pragma unroll
    for (int C = 0; C < kC; ++C)
#pragma unroll
      for (int e = 0; e < 2; ++e)
        qf[C][e] = *reinterpret_cast<const half8*>(qrow + 64 * C + 16 * quad + 8 * e);

    float4v o[kT];
#pragma unroll
    for (int t = 0; t < kT; ++t) o[t] = float4v{0, 0, 0, 0};
    float m = -INFINITY, l = 0.0f, unit = 1.0f;

    for (int i = begin + wave; i < end; i += 4) {
      const int blk = vis.page(i);
      const int page = a.table[(int64_t)b * a.max_pages + blk];
      if ((uint32_t)page >= (uint32_t)a.num_pages) continue;
      const int64_t at = (int64_t)page * a.kv_heads + head;
      const uint8_t* const kp = a.k_pages + at * (kPage * D);
      const uint8_t* const vp = a.v_pages + at * (kPage * D);
      const float ks = a.scale_log2 * a.k_scales[at], vs = a.v_scales[at];

      // S^T: row m of tile t4 is token 16 (m / 4) + 4 t4 + m % 4, so that lane
      // (col, quad) ends with tokens 16 quad + 4 t4 + i.
      float s[16];
#pragma unroll
      for (int t4 = 0; t4 < 4; ++t4) {
        float4v acc = {0, 0, 0, 0};
        const uint8_t* const krow = kp + (16 * (col >> 2) + 4 * t4 + (col & 3)) * D + 16 * quad;
#pragma unroll
        for (int C = 0; C < kC; ++C) {
          const uint4 kc = *reinterpret_cast<const uint4*>(krow + 64 * C);
          acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(codes8(kc.x, kc.y), qf[C][0], acc, 0, 0, 0);
          acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(codes8(kc.z, kc.w), qf[C][1], acc, 0, 0, 0);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) s[4 * t4 + e] = acc[e] * ks;
      }
      // Masks, where the page is not visible as a whole to every row.
      const int j0 = blk * kPage;
      if (!page_whole(j0, pmin, pmax, a.window, a.sinks)) {
#pragma unroll
        for (int e = 0; e < 16; ++e)
          s[e] = sees(pos, j0 + 16 * quad + e, a.window, a.sinks) ? s[e] : -INFINITY;
      }
      float top = s[0];
#pragma unroll
      for (int e = 1; e < 16; ++e) top = fmaxf(top, s[e]);
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      const float m_new = fmaxf(m, top);
      const float base = m_new == -INFINITY ? 0.0f : m_new;
      const float alpha = exp2_hw(m - base);
      m = m_new;
      l *= alpha;
      half8 p[2];
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const float x = exp2_hw(s[e] - base);
        l += x;
        p[e / 8][e % 8] = (_Float16)x;
      }
      const float fix = alpha * (unit / vs);
      unit = vs;
      // O^T: lane (col, quad) gives channel 16 t + col of tokens 16 quad and
      // up.  Slots past the sequence's end may hold anything: no NaN of theirs
      // may meet the zero weight.
      const int held = seq.length - j0 - 16 * quad;   // valid slots of this lane's 16
#pragma unroll
      for (int t = 0; t < kT; ++t) {
        uint4 vc = *reinterpret_cast<const uint4*>(vp + (16 * t + col) * kPage + 16 * quad);
        if (j0 + kPage > seq.length) {
          uint32_t* const w = &vc.x;
#pragma unroll
          for (int d = 0; d < 4; ++d) w[d] &= held_mask(held, 4 * d);
        }
        o[t] *= fix;
        o[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(codes8(vc.x, vc.y), p[0], o[t], 0, 0, 0);
        o[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(codes8(vc.z, vc.w), p[1], o[t], 0, 0, 0);
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
    for (int w = 0; w < 4; ++w) {
      if (w == wave) {
#pragma unroll
        for (int t = 0; t < kT; ++t) {
          float4v* const dst = reinterpret_cast<float4v*>(sum_o + col * D + 16 * t + 4 * quad);
          *dst = w == 0 ? o[t] * mine : *dst + o[t] * mine;
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
      const int64_t to = ((int64_t)seq.first_row + r / a.group) * a.heads + head * a.group + r % a.group;
      if (a.splits == 1) {
        a.out[to * D + d] = __float2half_rn(ml.y > 0.0f ? sum_o[e] / ml.y : ml.y);
        if (d == 0) a.lse[to] = ml.x * kLn2 + logf(ml.y);
      } else {
        const int64_t at = (int64_t)blockIdx.z * a.T * a.heads + to;
        a.part_o[at * D + d] = sum_o[e];
        if (d == 0) a.part_ml[at] = ml;
      }
    }
    __syncthreads();
  }
}

// Joins the splits of one row: a wave a row.
template <int D>
__global__ void __launch_bounds__(256) kv8_combine_kernel(AttnArgs a) {
  const int64_t n = (int64_t)a.T * a.heads;
  const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (row >= n) return;
  const int lane = threadIdx.x & 63;
  float M = -INFINITY;
  for (int s = 0; s < a.splits; ++s) M = fmaxf(M, a.part_ml[s * n + row].x);
  const float ref = M == -INFINITY ? 0.0f : M;
  float L = 0.0f, o[D / 64] = {};
  for (int s = 0; s < a.splits; ++s) {
    const float2 ml = a.part_ml[s * n + row];
    const float f = exp2_hw(ml.x - ref);
    L += f * ml.y;
#pragma unroll
    for (int i = 0; i < D / 64; ++i) o[i] += f * a.part_o[(s * n + row) * D + 64 * i + lane];
  }
#pragma unroll
  for (int i = 0; i < D / 64; ++i) a.out[row * D + 64 * i + lane] = __float2half_rn(L > 0.0f ? o[i] / L : L);
  if (lane == 0) a.lse[row] = M * kLn2 + logf(L);
}

// Rows of a sequence's largest count that the tiles of 16 still take; more go
// to the tiles of kPromptRows.
constexpr int64_t kDecodeRows = 32;

bool is_prompt(const Kv8Attention& c) { return c.max_q * (c.heads / c.cache.kv_heads) > kDecodeRows; }

// Splits of the visible pages: enough workgroups for two on every compute
// unit, of four pages (one a wave) or more.
int choose_splits(const Kv8Attention& c) {
  const int64_t height = is_prompt(c) ? kPromptRows : 16;
  const int64_t tiles =
      ((c.max_q * (c.heads / c.cache.kv_heads) + height - 1) / height) * c.cache.B * c.cache.kv_heads;
  int64_t keys = c.max_len;
  if (c.window > 0 && (int64_t)c.window + c.sinks + c.max_q + 2 * kPage < keys)
    keys = (int64_t)c.window + c.sinks + c.max_q + 2 * kPage;
  const int64_t most = (keys + 4 * kPage - 1) / (4 * kPage);
  const int64_t want = (2 * (int64_t)device_cus() + tiles - 1) / tiles;
  const int64_t s = want < most ? want : most;
  return (int)(s < 1 ? 1 : s > 256 ? 256 : s);
}

template <int D>
hipError_t launch(const AttnArgs& a, const Kv8Attention& c, hipStream_t stream) {
  hipError_t e;
  if (is_prompt(c)) {
    e = launch_kv8_prompt(a, D, c.cache.B, c.max_q, stream);
  } else {
    const int64_t tiles = (c.max_q * a.group + 15) / 16;
    const dim3 grid((unsigned)(c.cache.B * a.kv_heads), (unsigned)(tiles < 65535 ? tiles : 65535),
                    (unsigned)a.splits);
    kv8_decode_kernel<D><<<grid, 256, 0, stream>>>(a);
    e = hipGetLastError();
  }
  if (e != hipSuccess || a.splits == 1) return e;
  kv8_combine_kernel<D><<<(unsigned)(((int64_t)a.T * a.heads + 3) / 4), 256, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace

int64_t kv8_attention_workspace(const Kv8Attention& c) {
  const int splits = choose_splits(c);
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
  a.max_pages = (int)c.cache.max_pages;
  a.num_pages = (int)c.cache.num_pages;
  a.heads = c.heads;
  a.kv_heads = c.cache.kv_heads;
  a.group = c.heads / c.cache.kv_heads;
  a.scale_log2 = c.scale * kLog2e;
  a.window = c.window;
  a.sinks = c.sinks;
  a.splits = choose_splits(c);
  a.out = static_cast<__half*>(c.out);
  a.lse = c.lse;
  a.part_o = static_cast<float*>(c.workspace);
  a.part_ml = reinterpret_cast<float2*>(a.part_o + (int64_t)a.splits * a.T * a.heads * c.cache.head_dim);
  switch (c.cache.head_dim) {
    case 64: return launch<64>(a, c, stream);
    case 128: return launch<128>(a, c, stream);
    case 256: return launch<256>(a, c, stream);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace dptq
