// What the two kernels of kv8_attention share: arguments, code conversion, the
// pages that a tile of queries sees.
#pragma once

#include "internal.h"
#include "kv8_device.h"

namespace dptq {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef float float4v __attribute__((ext_vector_type(4)));
typedef float float16v __attribute__((ext_vector_type(16)));

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

constexpr int kMaxSplits = 512;

struct AttnArgs {
  const __half* q;
  int64_t ld_q;
  const uint8_t *k_pages, *v_pages;
  const float *k_scales, *v_scales;
  const int32_t *cu, *lengths, *table;
  int T, max_pages, num_pages, heads, kv_heads, group;
  float scale_log2;        // scale * log2(e)
  int window, sinks;       // window 0: none
  int chunk, splits;       // pages of a part; the last part takes what is left
  __half* out;
  float* lse;
  float* part_o;           // [splits][T * heads][D], relative to their references
  float2* part_ml;         // [splits][T * heads] (reference, sum), base 2
};

__device__ __forceinline__ float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }

// Eight codes (two dwords) as halves.
__device__ __forceinline__ half8 codes8(uint32_t a, uint32_t b) {
  const half2v x0 = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, 1.0f, false);
  const half2v x1 = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, 1.0f, true);
  const half2v x2 = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, 1.0f, false);
  const half2v x3 = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, 1.0f, true);
  return half8{x0[0], x0[1], x1[0], x1[1], x2[0], x2[1], x3[0], x3[1]};
}

// Bytes of the dword of slots [first, first + 4) that lie below `held`.
__device__ __forceinline__ uint32_t held_mask(int held, int first) {
  const int n = held - first;
  return n >= 4 ? 0xFFFFFFFFu : n <= 0 ? 0u : (1u << (8 * n)) - 1u;
}

// Pages that a tile of rows with positions [pmin, pmax] reads: [0, sink_pages)
// and [first, last].
struct Visible {
  int sink_pages, first, total;
  __device__ int page(int i) const { return i < sink_pages ? i : first + (i - sink_pages); }
};

__device__ __forceinline__ Visible visible_pages(int pmin, int pmax, int window, int sinks, int max_pages) {
  if (pmax < 0 || max_pages == 0) return Visible{0, 0, 0};
  const int low = window > 0 ? max(pmin - window + 1, 0) : 0;
  const int last = min(pmax / kPage, max_pages - 1);
  const int sink_pages = window > 0 ? min((min(sinks, low) + kPage - 1) / kPage, last + 1) : 0;
  const int first = min(max(low / kPage, sink_pages), last + 1);   // last + 1: none (low may lie beyond the table)
  return Visible{sink_pages, first, sink_pages + last + 1 - first};
}

// Whether every row with positions in [pmin, pmax] sees the whole page from
// position j0; whether one of them sees any of it.
__device__ __forceinline__ bool page_whole(int j0, int pmin, int pmax, int window, int sinks) {
  return j0 + kPage - 1 <= pmin && (window == 0 || j0 > pmax - window || j0 + kPage <= sinks);
}
__device__ __forceinline__ bool page_any(int j0, int pmin, int pmax, int window, int sinks) {
  return j0 <= pmax && (window == 0 || j0 + kPage - 1 > pmin - window || j0 < sinks);
}

__device__ __forceinline__ bool sees(int pos, int j, int window, int sinks) {
  return j <= pos && (window == 0 || j > pos - window || j < sinks);
}

// Defined in kv8_prompt.hip; rows (query tokens x heads of a group) of a workgroup: 128 or 64.
hipError_t launch_kv8_prompt(const AttnArgs& a, int head_dim, int rows, int64_t B, int64_t max_q,
                             hipStream_t stream);

}  // namespace dptq
