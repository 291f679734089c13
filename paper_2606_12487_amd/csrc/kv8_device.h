// The 8-bit paged KV cache: geometry and code conversions shared by the
// kernels that write it (kv8_append.hip) and read it (kv8_attention.hip).
//
// A page holds 64 tokens of every KV head.  Per head, K codes are
// [64][head_dim] and V codes [head_dim][64]: a token of K and a channel of V
// are contiguous, which is how the matrix cores take them (both products of
// the attention sum over the contiguous index), so that the attention needs no
// transposition.  Codes are OCP e4m3; the value of a code is code * scale with
// one fp32 scale per page and head, for K and for V.
#pragma once

#include <hip/hip_runtime.h>
#include <hip/hip_fp16.h>
#include <stdint.h>

namespace dptq {

constexpr int kPage = 64;   // tokens of a page

// Smallest scale exponent; 448 * 2^-32 is below the smallest fp16 value.
constexpr int kKv8MinExp = -32;

// Where a sequence's new tokens lie: token row t of position p is
// first_row + (p - start), for start <= p < length and p >= 0.
struct KvSeq {
  int first_row, count, start, length;
};

// Offsets outside [0, T] are clamped to it; a sequence whose offsets run
// backwards has no tokens.
__device__ __forceinline__ KvSeq kv_seq(const int32_t* cu, const int32_t* lengths, int b, int T) {
  const int lo = min(max(cu[b], 0), T), hi = min(max(cu[b + 1], 0), T);
  const int count = max(hi - lo, 0), n = max(lengths[b], 0);
  return KvSeq{lo, count, n - count, n};
}

}  // namespace dptq
