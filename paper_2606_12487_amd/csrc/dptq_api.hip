// C ABI: argument checks, then dispatch to the gfx950 kernels.
#include "dptq.h"
#include "internal.h"
#include "rotary_device.h"

namespace {

using dptq::HadSplit;

constexpr int kVersion = 100;  // 0.1.0

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// h = 2^j or 28 * 2^j with h <= 32768.
bool split_had(int64_t h, HadSplit* out) {
  if (h < 1 || h > 32768) return false;
  if ((h & (h - 1)) == 0) {
    int j = 0;
    while ((int64_t{1} << j) < h) ++j;
    *out = HadSplit{1, j};
    return true;
  }
  if (h % 28 == 0) {
    const int64_t p = h / 28;
    if ((p & (p - 1)) == 0) {
      int j = 0;
      while ((int64_t{1} << j) < p) ++j;
      *out = HadSplit{28, j};
      return true;
    }
  }
  return false;
}

int check_rotation_shape(int64_t M, int64_t K, int32_t had_size, HadSplit* hs) {
  if (M < 0 || K < 1) return DPTQ_ERR_INVALID_ARG;
  if (!split_had(had_size, hs)) return DPTQ_ERR_INVALID_ARG;
  if (K % had_size != 0 || K % 8 != 0) return DPTQ_ERR_INVALID_ARG;
  if (K > dptq::kMaxRotateK) return DPTQ_ERR_UNSUPPORTED;
  if (M > 0x7FFFFFFF) return DPTQ_ERR_UNSUPPORTED;
  return DPTQ_OK;
}

int check_gemm_shape(int64_t M, int64_t K, int32_t bits, int64_t N) {
  if (M < 0 || K < 1 || N < 1) return DPTQ_ERR_INVALID_ARG;
  if (bits != 4 && bits != 8) return DPTQ_ERR_INVALID_ARG;
  if (K % 128 != 0 || K > DPTQ_MAX_K) return DPTQ_ERR_UNSUPPORTED;
  if (N % 16 != 0 || N > 0x7FFFFFF0) return DPTQ_ERR_UNSUPPORTED;
  if (M > 0x7FFFFFFF) return DPTQ_ERR_UNSUPPORTED;
  if ((M > 16) && ((M + 127) / 128) * ((N + 255) / 256) > 0x7FFFFFFF) return DPTQ_ERR_UNSUPPORTED;
  return DPTQ_OK;
}

int from_hip(hipError_t e) { return e == hipSuccess ? DPTQ_OK : DPTQ_ERR_HIP; }

bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

// KV-cache shapes: group a power of two in [16, 512] dividing D; T * D < 2^40.
int check_kv_shape(int64_t T, int64_t D, int32_t group) {
  if (T < 0 || D < 1) return DPTQ_ERR_INVALID_ARG;
  if (group < 16 || group > 512 || (group & (group - 1)) != 0) return DPTQ_ERR_INVALID_ARG;
  if (D % group != 0) return DPTQ_ERR_INVALID_ARG;
  if (D > (int64_t{1} << 31) || T > (int64_t{1} << 40) / D) return DPTQ_ERR_UNSUPPORTED;
  return DPTQ_OK;
}

bool aligned8(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 7u) == 0; }

constexpr int64_t kMost30 = int64_t{1} << 30;

// Sizes of the 8-bit paged KV cache and of the sequences in it.
int check_kv8_shape(int64_t T, int64_t B, int64_t max_pages, int64_t num_pages, int32_t kv_heads,
                    int32_t head_dim) {
  if (T < 0 || B < 0 || max_pages < 0 || num_pages < 0 || kv_heads < 1 || head_dim < 1) return DPTQ_ERR_INVALID_ARG;
  if (head_dim != 64 && head_dim != 128 && head_dim != 256) return DPTQ_ERR_UNSUPPORTED;
  if (T >= kMost30 || B > 65535 || kv_heads > 1024) return DPTQ_ERR_UNSUPPORTED;
  if (max_pages > kMost30 / DPTQ_KV8_PAGE || num_pages > 0x7FFFFFFF) return DPTQ_ERR_UNSUPPORTED;
  return DPTQ_OK;
}

// Without pages, in the cache or in the table, nothing of either is read.
bool kv8_pointers(const dptq::Kv8Cache& c) {
  const bool pages = c.num_pages > 0 && c.max_pages > 0;
  if (pages && !(c.k_pages && c.v_pages && c.k_scales && c.v_scales && c.table)) return false;
  return c.cu && c.lengths && aligned16(c.k_pages) && aligned16(c.v_pages) && aligned4(c.k_scales) &&
         aligned4(c.v_scales) && aligned4(c.cu) && aligned4(c.lengths) && aligned4(c.table);
}

// Rows of n elements, ld apart, that 16-byte loads take.
bool rows_ok(const void* p, int64_t ld, int64_t n) { return p && aligned16(p) && ld >= n && ld % 8 == 0; }

// T rows of n fp16 elements, ld apart.
struct Rows {
  const void* p;
  int64_t ld, n;
};

// Whether no element is in a row of both.  Rows of equal distance are compared by
// where they stand in it; of unequal ones all between the first and the last
// element counts.
bool apart(const Rows& a, const Rows& b, int64_t T) {
  if (reinterpret_cast<uintptr_t>(a.p) > reinterpret_cast<uintptr_t>(b.p)) return apart(b, a, T);
  using wide = unsigned __int128;
  const wide d = reinterpret_cast<uintptr_t>(b.p) - reinterpret_cast<uintptr_t>(a.p);   // bytes
  const wide ld = 2 * (wide)a.ld, n_a = 2 * (wide)a.n, n_b = 2 * (wide)b.n;
  if (d >= (wide)(T - 1) * ld + n_a) return true;
  return T > 1 && a.ld == b.ld && d % ld >= n_a && ld - d % ld >= n_b;
}

// An output of rotary positions beside rows that are read: the same rows, or apart.
bool in_place_or_apart(const Rows& out, const Rows& in, int64_t T) {
  return (out.p == in.p && out.ld == in.ld && out.n == in.n) || apart(out, in, T);
}

// The sizes of a kv8_attention call; max_q and max_len within what T and the
// page table allow.
int attention_shape(int64_t T, int64_t B, int64_t max_pages, int64_t num_pages, int32_t heads, int32_t kv_heads,
                    int32_t head_dim, int32_t window, int32_t sinks, int64_t max_q, int64_t max_len,
                    dptq::Kv8Attention* c) {
  const int st = check_kv8_shape(T, B, max_pages, num_pages, kv_heads, head_dim);
  if (st != DPTQ_OK) return st;
  if (heads < 1 || heads % kv_heads != 0 || window < 0 || sinks < 0 || max_q < 0 || max_len < 0)
    return DPTQ_ERR_INVALID_ARG;
  if (window >= kMost30 || sinks >= kMost30 || heads > 65536 || T > kMost30 / heads) return DPTQ_ERR_UNSUPPORTED;
  const int64_t capacity = max_pages * DPTQ_KV8_PAGE;
  c->cache.T = T;
  c->cache.B = B;
  c->cache.max_pages = max_pages;
  c->cache.num_pages = num_pages;
  c->cache.kv_heads = kv_heads;
  c->cache.head_dim = head_dim;
  c->heads = heads;
  c->window = window;
  c->sinks = sinks;
  c->max_q = max_q > 0 && max_q < T ? max_q : T;
  c->max_len = max_len > 0 && max_len < capacity ? max_len : capacity;
  return DPTQ_OK;
}

// The gated epilogue of an activation: sigmoid's argument is g (c1 + c2 g^2), in
// powers of two.
bool gate_of(int32_t act, dptq::Gate* gate) {
  constexpr double kLog2e = 1.4426950408889634, kC1 = 1.5957691216057308;   // 2 sqrt(2 / pi)
  if (act == DPTQ_GATE_SILU) *gate = dptq::Gate{(float)-kLog2e, 0.0f};
  else if (act == DPTQ_GATE_GELU_TANH) *gate = dptq::Gate{(float)(-kLog2e * kC1), (float)(-kLog2e * kC1 * 0.044715)};
  else return false;
  return true;
}

// Sizes of a gated block: those of dptq_qlinear with 2 F rows of weights.
int check_gated_shape(int64_t M, int64_t K, int32_t bits, int64_t F) {
  if (F < 1 || F % 8 != 0) return DPTQ_ERR_INVALID_ARG;
  if (F > 0x3FFFFFF8) return DPTQ_ERR_UNSUPPORTED;
  return check_gemm_shape(M, K, bits, 2 * F);
}

// What rotary positions add to the check of a call.
int check_rotary(int32_t heads, int32_t kv_heads, int32_t head_dim, int32_t rotary_dim, float scale) {
  if (heads < 1 || kv_heads < 0 || head_dim < 1 || head_dim % 8 != 0) return DPTQ_ERR_INVALID_ARG;
  if (rotary_dim < 2 || rotary_dim % 2 != 0 || rotary_dim > head_dim) return DPTQ_ERR_INVALID_ARG;
  if (!(scale >= -3.0e38f && scale <= 3.0e38f)) return DPTQ_ERR_INVALID_ARG;   // also rejects NaN
  if (head_dim > dptq::kMaxRotaryHead || heads > 8192 || kv_heads > 8192 - heads) return DPTQ_ERR_UNSUPPORTED;
  return DPTQ_OK;
}

int logprobs_shape(int64_t ld, int64_t M, int64_t V, int32_t top, int32_t dtype, dptq::TokenLogprobs* c) {
  if (M < 0 || V < 1 || top < 0 || top > V || ld < V) return DPTQ_ERR_INVALID_ARG;
  if (dtype != DPTQ_F16 && dtype != DPTQ_F32) return DPTQ_ERR_INVALID_ARG;
  if (M > 0x7FFFFFFF || V >= kMost30 || top > DPTQ_MAX_TOP) return DPTQ_ERR_UNSUPPORTED;
  c->fp32 = dtype == DPTQ_F32;
  c->ld = ld;
  c->M = M;
  c->V = (int)V;
  c->top = top;
  return DPTQ_OK;
}

int sample_shape(int64_t ld, int64_t M, int64_t V, int32_t dtype, dptq::SampleTokens* c) {
  dptq::TokenLogprobs l{};   // the same rows
  const int st = logprobs_shape(ld, M, V, 0, dtype, &l);
  c->fp32 = l.fp32;
  c->ld = l.ld;
  c->M = l.M;
  c->V = l.V;
  return st;
}

}  // namespace

extern "C" {

const char* dptq_status_string(int status) {
  switch (status) {
    case DPTQ_OK: return "ok";
    case DPTQ_ERR_INVALID_ARG: return "invalid argument";
    case DPTQ_ERR_UNSUPPORTED: return "unsupported shape or size";
    case DPTQ_ERR_HIP: return "HIP runtime error";
    default: return "unknown status";
  }
}

int dptq_version(void) { return kVersion; }

int dptq_rotate_quant(const void* x, int64_t M, int64_t K, int32_t had_size, int32_t bits,
                      void* codes, float* a_scales, void* stream) {
  HadSplit hs{};
  int st = check_rotation_shape(M, K, had_size, &hs);
  if (st != DPTQ_OK) return st;
  if (bits != 4 && bits != 8) return DPTQ_ERR_INVALID_ARG;
  if (M == 0) return DPTQ_OK;
  if (!x || !codes || !a_scales) return DPTQ_ERR_INVALID_ARG;
  if (!aligned16(x) || !aligned16(codes) || !aligned16(a_scales)) return DPTQ_ERR_INVALID_ARG;
  return from_hip(dptq::launch_rotate_quant_f16(x, M, (int)K, hs, bits, codes, a_scales,
                                                static_cast<hipStream_t>(stream)));
}

int dptq_qlinear(const void* codes, const float* a_scales, int64_t M, int64_t K, int32_t bits,
                 const uint8_t* w_packed, const float* w_scales, int64_t N, void* y,
                 void* stream) {
  int st = check_gemm_shape(M, K, bits, N);
  if (st != DPTQ_OK) return st;
  if (M == 0) return DPTQ_OK;
  if (!codes || !a_scales || !w_packed || !w_scales || !y) return DPTQ_ERR_INVALID_ARG;
  if (!aligned16(codes) || !aligned16(a_scales) || !aligned16(w_packed) ||
      !aligned16(w_scales) || !aligned16(y))
    return DPTQ_ERR_INVALID_ARG;
  return from_hip(dptq::launch_qlinear(codes, a_scales, M, (int)K, bits, w_packed, w_scales, N,
                                       y, nullptr, dptq::kGemmAuto, static_cast<hipStream_t>(stream)));
}

int dptq_qlinear_acc(const void* codes, int64_t M, int64_t K, int32_t bits,
                     const uint8_t* w_packed, int64_t N, int32_t* acc, void* stream) {
  int st = check_gemm_shape(M, K, bits, N);
  if (st != DPTQ_OK) return st;
  if (M == 0) return DPTQ_OK;
  if (!codes || !w_packed || !acc) return DPTQ_ERR_INVALID_ARG;
  if (!aligned16(codes) || !aligned16(w_packed) || !aligned16(acc)) return DPTQ_ERR_INVALID_ARG;
  return from_hip(dptq::launch_qlinear(codes, nullptr, M, (int)K, bits, w_packed, nullptr, N,
                                       nullptr, acc, dptq::kGemmAuto, static_cast<hipStream_t>(stream)));
}

int dptq_residual_dynamics(const void* x, const void* dx, int64_t T, int64_t K, int32_t had_size,
                           int32_t bits, float eps, float* jr, float* snr, double* layer_means,
                           void* stream) {
  HadSplit hs{};
  int st = check_rotation_shape(T, K, had_size, &hs);
  if (st != DPTQ_OK) return st;
  if (bits != 4 && bits != 8) return DPTQ_ERR_INVALID_ARG;
  if (!(eps >= 0.0f) || eps > 3.0e38f) return DPTQ_ERR_INVALID_ARG;   // also rejects NaN
  if (T == 0) return DPTQ_OK;
  if (!x || !dx || !jr || !snr) return DPTQ_ERR_INVALID_ARG;
  if (!aligned16(x) || !aligned16(dx)) return DPTQ_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(jr) & 3u) || (reinterpret_cast<uintptr_t>(snr) & 3u) ||
      (reinterpret_cast<uintptr_t>(layer_means) & 7u))
    return DPTQ_ERR_INVALID_ARG;
  return from_hip(dptq::launch_residual_stats(x, dx, T, (int)K, hs, bits, eps, jr, snr,
                                              layer_means, static_cast<hipStream_t>(stream)));
}

int dptq_select_layers(int32_t num_layers, const double* jr, const double* snr, double tau_jr,
                       double tau_snr, int32_t* bits_out) {
  if (num_layers < 1 || !jr || !snr || !bits_out) return DPTQ_ERR_INVALID_ARG;
  for (int32_t l = 0; l < num_layers; ++l)
    bits_out[l] = (jr[l] > tau_jr && snr[l] < tau_snr) ? 8 : 4;
  return DPTQ_OK;
}

int dptq_kv_quant(const void* kv, int64_t T, int64_t D, int32_t group, uint8_t* codes,
                  float* scales, float* mins, void* stream) {
  const int st = check_kv_shape(T, D, group);
  if (st != DPTQ_OK) return st;
  if (T == 0) return DPTQ_OK;
  if (!kv || !codes || !scales || !mins) return DPTQ_ERR_INVALID_ARG;
  if (!aligned16(kv) || !aligned4(codes) || !aligned4(scales) || !aligned4(mins))
    return DPTQ_ERR_INVALID_ARG;
  return from_hip(dptq::launch_kv_quant(kv, T, D, group, codes, scales, mins,
                                        static_cast<hipStream_t>(stream)));
}

int dptq_kv_dequant(const uint8_t* codes, const float* scales, const float* mins, int64_t T,
                    int64_t D, int32_t group, void* kv_out, void* stream) {
  const int st = check_kv_shape(T, D, group);
  if (st != DPTQ_OK) return st;
  if (T == 0) return DPTQ_OK;
  if (!kv_out || !codes || !scales || !mins) return DPTQ_ERR_INVALID_ARG;
  if (!aligned16(kv_out) || !aligned4(codes) || !aligned4(scales) || !aligned4(mins))
    return DPTQ_ERR_INVALID_ARG;
  return from_hip(dptq::launch_kv_dequant(codes, scales, mins, T, D, group, kv_out,
                                          static_cast<hipStream_t>(stream)));
}

int dptq_qlinear_kernel(const void* codes, const float* a_scales, int64_t M, int64_t K,
                        int32_t bits, const uint8_t* w_packed, const float* w_scales,
                        int64_t N, void* y, int32_t* acc, int32_t kernel, void* stream) {
  int st = check_gemm_shape(M, K, bits, N);
  if (st != DPTQ_OK) return st;
  if (kernel < DPTQ_GEMM_AUTO || kernel > DPTQ_GEMM_TILE_192X256) return DPTQ_ERR_INVALID_ARG;
  if ((y == nullptr) == (acc == nullptr)) return DPTQ_ERR_INVALID_ARG;
  if (!dptq::gemm_kernel_fits(kernel, M, N, (int)K, bits)) return DPTQ_ERR_UNSUPPORTED;
  if (M == 0) return DPTQ_OK;
  if (!codes || !w_packed) return DPTQ_ERR_INVALID_ARG;
  if (!aligned16(codes) || !aligned16(w_packed)) return DPTQ_ERR_INVALID_ARG;
  if (y) {
    if (!a_scales || !w_scales) return DPTQ_ERR_INVALID_ARG;
    if (!aligned16(a_scales) || !aligned16(w_scales) || !aligned16(y)) return DPTQ_ERR_INVALID_ARG;
    return from_hip(dptq::launch_qlinear(codes, a_scales, M, (int)K, bits, w_packed, w_scales, N,
                                         y, nullptr, kernel, static_cast<hipStream_t>(stream)));
  }
  if (!aligned16(acc)) return DPTQ_ERR_INVALID_ARG;
  return from_hip(dptq::launch_qlinear(codes, nullptr, M, (int)K, bits, w_packed, nullptr, N,
                                       nullptr, acc, kernel, static_cast<hipStream_t>(stream)));
}

int dptq_pack_w4_a8(const uint8_t* w_packed, int64_t N, int64_t K, uint8_t* out, void* stream) {
  if (N < 0 || K < 1) return DPTQ_ERR_INVALID_ARG;
  if (K % 128 != 0 || K > DPTQ_MAX_K || N > 0x7FFFFFF0) return DPTQ_ERR_UNSUPPORTED;
  if (N == 0) return DPTQ_OK;
  if (!w_packed || !out) return DPTQ_ERR_INVALID_ARG;
  if (!aligned16(w_packed) || !aligned16(out)) return DPTQ_ERR_INVALID_ARG;
  return from_hip(dptq::launch_pack_w4_a8(w_packed, N, (int)K, out, static_cast<hipStream_t>(stream)));
}

int dptq_qlinear_a8(const void* codes, const float* a_scales, int64_t M, int64_t K,
                    const uint8_t* w_a8, const float* w_scales, int64_t N, void* y, int32_t kernel,
                    void* stream) {
  int st = check_gemm_shape(M, K, 8, N);
  if (st != DPTQ_OK) return st;
  if (kernel < DPTQ_GEMM_AUTO || kernel > DPTQ_GEMM_TILE_192X256) return DPTQ_ERR_INVALID_ARG;
  if (!dptq::gemm_kernel_fits(kernel, M, N, (int)K, 8)) return DPTQ_ERR_UNSUPPORTED;
  if (M == 0) return DPTQ_OK;
  if (!codes || !a_scales || !w_a8 || !w_scales || !y) return DPTQ_ERR_INVALID_ARG;
  if (!aligned16(codes) || !aligned16(a_scales) || !aligned16(w_a8) || !aligned16(w_scales) ||
      !aligned16(y))
    return DPTQ_ERR_INVALID_ARG;
  return from_hip(dptq::launch_qlinear_a8(codes, a_scales, M, (int)K, w_a8, w_scales, N, y, kernel,
                                          static_cast<hipStream_t>(stream)));
}

int64_t dptq_fp6_bytes(int64_t rows, int64_t K) {
  if (rows < 0 || K < 128 || K % 128 != 0 || K > DPTQ_MAX_K || rows > 0x7FFFFFFF) return -1;
  return dptq::fp6_bytes(rows, K);
}

int dptq_pack_fp6(const uint8_t* codes, int64_t rows, int64_t K, uint8_t* out, void* stream) {
  if (rows < 0 || K < 1) return DPTQ_ERR_INVALID_ARG;
  if (K % 128 != 0 || K > DPTQ_MAX_K || rows > 0x7FFFFFFF) return DPTQ_ERR_UNSUPPORTED;
  if (rows == 0) return DPTQ_OK;
  if (!codes || !out) return DPTQ_ERR_INVALID_ARG;
  if (!aligned16(codes) || !aligned16(out)) return DPTQ_ERR_INVALID_ARG;
  return from_hip(dptq::launch_pack_fp6(codes, rows, (int)K, out, static_cast<hipStream_t>(stream)));
}

int64_t dptq_prepacked_bytes(int64_t N, int64_t K, int32_t layout) {
  if (N < 0 || K < 128 || K % 128 != 0 || K > DPTQ_MAX_K) return -1;
  if (layout == DPTQ_WEIGHTS_FP6) return dptq_fp6_bytes(N, K);
  if (layout == DPTQ_WEIGHTS_A8_ORDER) return N > 0x7FFFFFF0 ? -1 : N * (K / 2);
  if (layout == DPTQ_WEIGHTS_DECODE) return (N > 0x7FFFFFF0 || N % 16 != 0) ? -1 : N * (K / 2);
  return -1;
}

int dptq_prepack_weights(const uint8_t* w_packed, int64_t N, int64_t K, int32_t layout,
                         uint8_t* w_native, void* stream) {
  if (layout == DPTQ_WEIGHTS_FP6) return dptq_pack_fp6(w_packed, N, K, w_native, stream);
  if (layout == DPTQ_WEIGHTS_A8_ORDER) return dptq_pack_w4_a8(w_packed, N, K, w_native, stream);
  if (layout == DPTQ_WEIGHTS_DECODE) {
    if (N < 0 || K < 1) return DPTQ_ERR_INVALID_ARG;
    if (K % 128 != 0 || K > DPTQ_MAX_K || N > 0x7FFFFFF0 || N % 16 != 0) return DPTQ_ERR_UNSUPPORTED;
    if (N == 0) return DPTQ_OK;
    if (!w_packed || !w_native) return DPTQ_ERR_INVALID_ARG;
    if (!aligned16(w_packed) || !aligned16(w_native)) return DPTQ_ERR_INVALID_ARG;
    return from_hip(dptq::launch_pack_decode(w_packed, N, (int)K, w_native,
                                             static_cast<hipStream_t>(stream)));
  }
  return DPTQ_ERR_INVALID_ARG;
}

int dptq_qlinear_decode_native(const void* codes, const float* a_scales, int64_t M, int64_t K,
                               int32_t bits, const uint8_t* w_dec, const float* w_scales,
                               int64_t N, void* y, int32_t* acc, void* stream) {
  int st = check_gemm_shape(M, K, bits, N);
  if (st != DPTQ_OK) return st;
  if (M > 16) return DPTQ_ERR_UNSUPPORTED;
  if ((y == nullptr) == (acc == nullptr)) return DPTQ_ERR_INVALID_ARG;
  if (M == 0) return DPTQ_OK;
  if (!codes || !w_dec) return DPTQ_ERR_INVALID_ARG;
  if (!aligned16(codes) || !aligned16(w_dec)) return DPTQ_ERR_INVALID_ARG;
  if (y) {
    if (!a_scales || !w_scales) return DPTQ_ERR_INVALID_ARG;
    if (!aligned16(a_scales) || !aligned16(w_scales) || !aligned16(y)) return DPTQ_ERR_INVALID_ARG;
  } else if (!aligned16(acc)) {
    return DPTQ_ERR_INVALID_ARG;
  }
  return from_hip(dptq::launch_qlinear_decode_native(codes, y ? a_scales : nullptr, M, (int)K, bits,
                                                     w_dec, y ? w_scales : nullptr, N, y,
                                                     y ? nullptr : acc,
                                                     static_cast<hipStream_t>(stream)));
}

int dptq_rotate_quant_fp6(const void* x, int64_t M, int64_t K, int32_t had_size, uint8_t* out,
                          float* a_scales, void* stream) {
  HadSplit hs{};
  int st = check_rotation_shape(M, K, had_size, &hs);
  if (st != DPTQ_OK) return st;
  if (K % 128 != 0) return DPTQ_ERR_UNSUPPORTED;
  if (M == 0) return DPTQ_OK;
  if (!x || !out || !a_scales) return DPTQ_ERR_INVALID_ARG;
  if (!aligned16(x) || !aligned16(out) || !aligned16(a_scales)) return DPTQ_ERR_INVALID_ARG;
  return from_hip(dptq::launch_rotate_quant_fp6(x, M, (int)K, hs, out, a_scales,
                                                static_cast<hipStream_t>(stream)));
}

int dptq_rotate_quant_ex(const void* x, int64_t M, int64_t K, int32_t had_size, int32_t bits,
                         const uint8_t* signs, int32_t layout, void* out, float* a_scales,
                         void* stream) {
  HadSplit hs{};
  int st = check_rotation_shape(M, K, had_size, &hs);
  if (st != DPTQ_OK) return st;
  if (bits != 4 && bits != 8) return DPTQ_ERR_INVALID_ARG;
  if (layout != DPTQ_LAYOUT_PACKED && layout != DPTQ_LAYOUT_FP6) return DPTQ_ERR_INVALID_ARG;
  if (layout == DPTQ_LAYOUT_FP6 && bits != 4) return DPTQ_ERR_INVALID_ARG;
  if (layout == DPTQ_LAYOUT_FP6 && K % 128 != 0) return DPTQ_ERR_UNSUPPORTED;
  if (M == 0) return DPTQ_OK;
  if (!x || !out || !a_scales) return DPTQ_ERR_INVALID_ARG;
  if (!aligned16(x) || !aligned16(out) || !aligned16(a_scales)) return DPTQ_ERR_INVALID_ARG;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  if (layout == DPTQ_LAYOUT_FP6)
    return from_hip(dptq::launch_rotate_quant_fp6(x, M, (int)K, hs, static_cast<uint8_t*>(out),
                                                  a_scales, s, signs));
  return from_hip(dptq::launch_rotate_quant_signed(x, M, (int)K, hs, bits, signs, out, a_scales, s));
}

int dptq_prepare_weights_signed(const float* w, int64_t N, int64_t K, int32_t had_size,
                                const uint8_t* signs, uint8_t* w_packed, float* w_scales,
                                void* stream) {
  HadSplit hs{};
  int st = check_rotation_shape(N, K, had_size, &hs);
  if (st != DPTQ_OK) return st;
  if (N == 0) return DPTQ_OK;
  if (!w || !w_packed || !w_scales) return DPTQ_ERR_INVALID_ARG;
  if (!aligned16(w) || !aligned16(w_packed) || !aligned16(w_scales)) return DPTQ_ERR_INVALID_ARG;
  return from_hip(dptq::launch_prepare_weights(w, N, (int)K, hs, w_packed, w_scales,
                                               static_cast<hipStream_t>(stream), signs));
}

int dptq_qlinear_fp6(const uint8_t* a_fp6, const float* a_scales, int64_t M, int64_t K,
                     const uint8_t* w_fp6, const float* w_scales, int64_t N, void* y,
                     int32_t* acc, void* stream) {
  int st = check_gemm_shape(M, K, 4, N);
  if (st != DPTQ_OK) return st;
  if ((y == nullptr) == (acc == nullptr)) return DPTQ_ERR_INVALID_ARG;
  if (((M + 255) / 256) * ((N + 191) / 192) > 0x7FFFFFFF) return DPTQ_ERR_UNSUPPORTED;
  if (M == 0) return DPTQ_OK;
  if (!a_fp6 || !w_fp6) return DPTQ_ERR_INVALID_ARG;
  if (!aligned16(a_fp6) || !aligned16(w_fp6)) return DPTQ_ERR_INVALID_ARG;
  if (y) {
    if (!a_scales || !w_scales) return DPTQ_ERR_INVALID_ARG;
    if (!aligned4(a_scales) || !aligned4(w_scales) || !aligned16(y)) return DPTQ_ERR_INVALID_ARG;
  } else if (!aligned16(acc)) {
    return DPTQ_ERR_INVALID_ARG;
  }
  return from_hip(dptq::launch_qlinear_fp6(a_fp6, y ? a_scales : nullptr, M, (int)K, w_fp6,
                                           y ? w_scales : nullptr, N, y, y ? nullptr : acc,
                                           static_cast<hipStream_t>(stream)));
}

int dptq_qlinear_gated(const void* codes, const float* a_scales, int64_t M, int64_t K, int32_t bits,
                       const uint8_t* w, int32_t weights, const float* w_scales, int64_t F, int32_t act,
                       void* y, void* stream) {
  const int st = check_gated_shape(M, K, bits, F);
  if (st != DPTQ_OK) return st;
  dptq::Gate gate{};
  if (!gate_of(act, &gate)) return DPTQ_ERR_INVALID_ARG;
  if (weights != DPTQ_WEIGHTS_PACKED && weights != DPTQ_WEIGHTS_A8_ORDER && weights != DPTQ_WEIGHTS_DECODE)
    return DPTQ_ERR_INVALID_ARG;
  if (weights == DPTQ_WEIGHTS_A8_ORDER && bits != 8) return DPTQ_ERR_INVALID_ARG;
  if (weights == DPTQ_WEIGHTS_DECODE && M > 16) return DPTQ_ERR_UNSUPPORTED;
  if (M == 0) return DPTQ_OK;
  if (!codes || !a_scales || !w || !w_scales || !y) return DPTQ_ERR_INVALID_ARG;
  if (!aligned16(codes) || !aligned16(a_scales) || !aligned16(w) || !aligned16(w_scales) || !aligned16(y))
    return DPTQ_ERR_INVALID_ARG;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  if (weights == DPTQ_WEIGHTS_DECODE)
    return from_hip(dptq::launch_qlinear_decode_native(codes, a_scales, M, (int)K, bits, w, w_scales, 2 * F, y, nullptr,
                                                       s, &gate));
  return from_hip(dptq::launch_qlinear_gated(codes, a_scales, M, (int)K, bits, w, w_scales, 2 * F, y, weights, gate, s));
}

int dptq_qlinear_gated_fp6(const uint8_t* a_fp6, const float* a_scales, int64_t M, int64_t K,
                           const uint8_t* w_fp6, const float* w_scales, int64_t F, int32_t act, void* y,
                           void* stream) {
  const int st = check_gated_shape(M, K, 4, F);
  if (st != DPTQ_OK) return st;
  dptq::Gate gate{};
  if (!gate_of(act, &gate)) return DPTQ_ERR_INVALID_ARG;
  if (((M + 255) / 256) * ((2 * F + 191) / 192) > 0x7FFFFFFF) return DPTQ_ERR_UNSUPPORTED;
  if (M == 0) return DPTQ_OK;
  if (!a_fp6 || !a_scales || !w_fp6 || !w_scales || !y) return DPTQ_ERR_INVALID_ARG;
  if (!aligned16(a_fp6) || !aligned16(w_fp6) || !aligned4(a_scales) || !aligned4(w_scales) || !aligned16(y))
    return DPTQ_ERR_INVALID_ARG;
  return from_hip(dptq::launch_qlinear_fp6(a_fp6, a_scales, M, (int)K, w_fp6, w_scales, 2 * F, y, nullptr,
                                           static_cast<hipStream_t>(stream), &gate));
}

int dptq_qlinear_decode_fused(const void* x, int64_t M, int64_t K, int32_t had_size,
                              int32_t bits, const uint8_t* w_packed, const float* w_scales,
                              int64_t N, void* y, void* codes, float* a_scales, int32_t mode,
                              void* stream) {
  HadSplit hs{};
  int st = check_rotation_shape(M, K, had_size, &hs);
  if (st != DPTQ_OK) return st;
  st = check_gemm_shape(M, K, bits, N);
  if (st != DPTQ_OK) return st;
  if (mode < DPTQ_DECODE_AUTO || mode > DPTQ_DECODE_TWO_LAUNCHES) return DPTQ_ERR_INVALID_ARG;
  if (M > 16) return DPTQ_ERR_UNSUPPORTED;
  if (mode == DPTQ_DECODE_ONE_LAUNCH && dptq::decode_fused_lds(M, (int)K, hs, bits) > dptq::kFusedLdsMax)
    return DPTQ_ERR_UNSUPPORTED;
  if (M == 0) return DPTQ_OK;
  if (!x || !w_packed || !w_scales || !y || !codes || !a_scales) return DPTQ_ERR_INVALID_ARG;
  if (!aligned16(x) || !aligned16(w_packed) || !aligned16(w_scales) || !aligned16(y) ||
      !aligned16(codes) || !aligned16(a_scales))
    return DPTQ_ERR_INVALID_ARG;
  return from_hip(dptq::launch_decode_fused(x, M, (int)K, hs, bits, w_packed, w_scales, N, y, codes,
                                            a_scales, mode, static_cast<hipStream_t>(stream)));
}

int dptq_rotate_quant_range(const void* x, int64_t M, int64_t K, int32_t had_size, int32_t bits,
                            void* codes, float* a_scales, int32_t* a_zeros, void* stream) {
  HadSplit hs{};
  int st = check_rotation_shape(M, K, had_size, &hs);
  if (st != DPTQ_OK) return st;
  if (bits != 4 && bits != 8) return DPTQ_ERR_INVALID_ARG;
  if (K % 128 != 0) return DPTQ_ERR_UNSUPPORTED;
  if (M == 0) return DPTQ_OK;
  if (!x || !codes || !a_scales || !a_zeros) return DPTQ_ERR_INVALID_ARG;
  if (!aligned16(x) || !aligned16(codes) || !aligned4(a_scales) || !aligned4(a_zeros))
    return DPTQ_ERR_INVALID_ARG;
  return from_hip(dptq::launch_rotate_quant_range(x, M, (int)K, hs, bits, codes, a_scales, a_zeros,
                                                  static_cast<hipStream_t>(stream)));
}

int dptq_weight_sums(const uint8_t* w_packed, int64_t N, int64_t K, int32_t* w_sums, void* stream) {
  if (N < 0 || K < 1) return DPTQ_ERR_INVALID_ARG;
  if (K % 32 != 0 || K > DPTQ_MAX_K || N > 0x7FFFFFF0) return DPTQ_ERR_UNSUPPORTED;
  if (N == 0) return DPTQ_OK;
  if (!w_packed || !w_sums || !aligned16(w_packed) || !aligned4(w_sums)) return DPTQ_ERR_INVALID_ARG;
  return from_hip(dptq::launch_weight_sums(w_packed, N, (int)K, w_sums,
                                           static_cast<hipStream_t>(stream)));
}

int dptq_qlinear_range(const void* codes, const float* a_scales, const int32_t* a_zeros, int64_t M,
                       int64_t K, int32_t bits, const uint8_t* w_packed, const float* w_scales,
                       const int32_t* w_sums, int64_t N, void* y, void* stream) {
  int st = check_gemm_shape(M, K, bits, N);
  if (st != DPTQ_OK) return st;
  if (M == 0) return DPTQ_OK;
  if (!codes || !a_scales || !a_zeros || !w_packed || !w_scales || !w_sums || !y)
    return DPTQ_ERR_INVALID_ARG;
  if (!aligned16(codes) || !aligned16(a_scales) || !aligned4(a_zeros) || !aligned16(w_packed) ||
      !aligned16(w_scales) || !aligned16(w_sums) || !aligned16(y))
    return DPTQ_ERR_INVALID_ARG;
  return from_hip(dptq::launch_qlinear_zp(codes, a_scales, a_zeros, M, (int)K, bits, w_packed, w_scales,
                                          w_sums, N, y, static_cast<hipStream_t>(stream)));
}

int dptq_rms_norm_quant(const void* x, const void* residual, const void* weight, int64_t M, int64_t K,
                        float eps, void* sum, int8_t* codes, float* scales, void* stream) {
  if (M < 0 || K < 1 || K % 8 != 0) return DPTQ_ERR_INVALID_ARG;
  if (!(eps >= 0.0f) || eps > 3.0e38f) return DPTQ_ERR_INVALID_ARG;   // also rejects NaN
  if (K > 65536 || M > 0x7FFFFFFF) return DPTQ_ERR_UNSUPPORTED;
  if (M == 0) return DPTQ_OK;
  if (!x || !weight || !codes || !scales || (residual == nullptr) != (sum == nullptr)) return DPTQ_ERR_INVALID_ARG;
  if (!aligned16(x) || !aligned16(residual) || !aligned16(weight) || !aligned16(sum) || !aligned16(codes) ||
      !aligned4(scales))
    return DPTQ_ERR_INVALID_ARG;
  return from_hip(dptq::launch_rms_norm_quant(x, residual, weight, M, (int)K, eps, sum, codes, scales,
                                              static_cast<hipStream_t>(stream)));
}

int dptq_kv8_append(const void* k, int64_t ld_k, const void* v, int64_t ld_v, int64_t T,
                    const int32_t* cu_seqlens, const int32_t* lengths, int64_t B,
                    const int32_t* page_table, int64_t max_pages, int64_t num_pages, int32_t kv_heads,
                    int32_t head_dim, uint8_t* k_pages, uint8_t* v_pages, float* k_scales,
                    float* v_scales, int64_t max_new, void* stream) {
  const int st = check_kv8_shape(T, B, max_pages, num_pages, kv_heads, head_dim);
  if (st != DPTQ_OK) return st;
  if (max_new < 0) return DPTQ_ERR_INVALID_ARG;
  if (T == 0 || B == 0 || max_pages == 0 || num_pages == 0) return DPTQ_OK;
  const dptq::Kv8Cache c{k_pages, v_pages, k_scales, v_scales, cu_seqlens, lengths, page_table,
                         T, B, max_pages, num_pages, kv_heads, head_dim};
  const int64_t row = (int64_t)kv_heads * head_dim;
  if (!kv8_pointers(c) || !rows_ok(k, ld_k, row) || !rows_ok(v, ld_v, row)) return DPTQ_ERR_INVALID_ARG;
  return from_hip(dptq::launch_kv8_append(c, k, ld_k, v, ld_v, max_new > 0 && max_new < T ? max_new : T,
                                          static_cast<hipStream_t>(stream)));
}

int dptq_rotary(const void* q, int64_t ld_q, int32_t heads, const void* k, int64_t ld_k, int32_t kv_heads,
                int64_t T, int32_t head_dim, const int32_t* positions, const double* inv_freq,
                int32_t rotary_dim, int32_t interleaved, float scale, void* q_out, int64_t ld_q_out,
                void* k_out, int64_t ld_k_out, void* stream) {
  const int st = check_rotary(heads, kv_heads, head_dim, rotary_dim, scale);
  if (st != DPTQ_OK) return st;
  if (T < 0) return DPTQ_ERR_INVALID_ARG;
  if (T >= kMost30) return DPTQ_ERR_UNSUPPORTED;
  if (T == 0) return DPTQ_OK;
  const int64_t row = (int64_t)heads * head_dim, kv_row = (int64_t)kv_heads * head_dim;
  if (!rows_ok(q, ld_q, row) || !rows_ok(q_out, ld_q_out, row)) return DPTQ_ERR_INVALID_ARG;
  if (kv_heads > 0 && (!rows_ok(k, ld_k, kv_row) || !rows_ok(k_out, ld_k_out, kv_row))) return DPTQ_ERR_INVALID_ARG;
  if (!positions || !inv_freq || !aligned4(positions) || !aligned8(inv_freq)) return DPTQ_ERR_INVALID_ARG;
  const Rows rq{q, ld_q, row}, rq_out{q_out, ld_q_out, row}, rk{k, ld_k, kv_row}, rk_out{k_out, ld_k_out, kv_row};
  if (!in_place_or_apart(rq_out, rq, T)) return DPTQ_ERR_INVALID_ARG;
  if (kv_heads > 0 && !(in_place_or_apart(rk_out, rk, T) && apart(rq_out, rk, T) && apart(rk_out, rq, T) &&
                        apart(rq_out, rk_out, T)))
    return DPTQ_ERR_INVALID_ARG;
  const dptq::RotaryCall c{q, k, q_out, k_out, ld_q, ld_k, ld_q_out, ld_k_out, T, heads, kv_heads,
                           head_dim, rotary_dim, positions, inv_freq, interleaved != 0, scale};
  return from_hip(dptq::launch_rotary(c, static_cast<hipStream_t>(stream)));
}

int dptq_rotary_kv8_append(const void* q, int64_t ld_q, int32_t heads, const void* k, int64_t ld_k,
                           const void* v, int64_t ld_v, int64_t T, const int32_t* cu_seqlens,
                           const int32_t* lengths, int64_t B, const int32_t* page_table,
                           int64_t max_pages, int64_t num_pages, int32_t kv_heads, int32_t head_dim,
                           uint8_t* k_pages, uint8_t* v_pages, float* k_scales, float* v_scales,
                           const double* inv_freq, int32_t rotary_dim, int32_t interleaved, float scale,
                           void* q_out, int64_t ld_q_out, int64_t max_new, void* stream) {
  int st = check_kv8_shape(T, B, max_pages, num_pages, kv_heads, head_dim);
  if (st == DPTQ_OK) st = check_rotary(heads, kv_heads, head_dim, rotary_dim, scale);
  if (st != DPTQ_OK) return st;
  if (max_new < 0) return DPTQ_ERR_INVALID_ARG;
  if (T == 0 || B == 0) return DPTQ_OK;
  const dptq::Kv8Cache c{k_pages, v_pages, k_scales, v_scales, cu_seqlens, lengths, page_table,
                         T, B, max_pages, num_pages, kv_heads, head_dim};
  const int64_t row = (int64_t)heads * head_dim, kv_row = (int64_t)kv_heads * head_dim;
  if (!kv8_pointers(c) || !rows_ok(k, ld_k, kv_row) || !rows_ok(v, ld_v, kv_row)) return DPTQ_ERR_INVALID_ARG;
  if (!rows_ok(q, ld_q, row) || !rows_ok(q_out, ld_q_out, row)) return DPTQ_ERR_INVALID_ARG;
  if (!inv_freq || !aligned8(inv_freq)) return DPTQ_ERR_INVALID_ARG;
  const Rows rq_out{q_out, ld_q_out, row};
  if (!in_place_or_apart(rq_out, Rows{q, ld_q, row}, T) || !apart(rq_out, Rows{k, ld_k, kv_row}, T) ||
      !apart(rq_out, Rows{v, ld_v, kv_row}, T))
    return DPTQ_ERR_INVALID_ARG;
  const dptq::RotaryCall r{q, k, q_out, nullptr, ld_q, ld_k, ld_q_out, 0, T, heads, kv_heads,
                           head_dim, rotary_dim, nullptr, inv_freq, interleaved != 0, scale};
  return from_hip(dptq::launch_rotary_kv8_append(c, r, v, ld_v, max_new > 0 && max_new < T ? max_new : T,
                                                 static_cast<hipStream_t>(stream)));
}

int64_t dptq_kv8_attention_workspace(int64_t T, int64_t B, int64_t max_pages, int32_t heads,
                                     int32_t kv_heads, int32_t head_dim, int32_t window, int32_t sinks,
                                     int64_t max_q, int64_t max_len) {
  dptq::Kv8Attention c{};
  if (attention_shape(T, B, max_pages, 1, heads, kv_heads, head_dim, window, sinks, max_q, max_len, &c) != DPTQ_OK)
    return -1;
  return T == 0 || B == 0 ? 0 : dptq::kv8_attention_workspace(c);
}

int dptq_kv8_attention(const void* q, int64_t ld_q, int64_t T, const int32_t* cu_seqlens,
                       const int32_t* lengths, int64_t B, const int32_t* page_table, int64_t max_pages,
                       int64_t num_pages, int32_t heads, int32_t kv_heads, int32_t head_dim,
                       const uint8_t* k_pages, const uint8_t* v_pages, const float* k_scales,
                       const float* v_scales, float scale, int32_t window, int32_t sinks,
                       int64_t max_q, int64_t max_len, void* out, float* lse, void* workspace,
                       int64_t workspace_bytes, void* stream) {
  dptq::Kv8Attention c{};
  const int st = attention_shape(T, B, max_pages, num_pages, heads, kv_heads, head_dim, window, sinks, max_q,
                                 max_len, &c);
  if (st != DPTQ_OK) return st;
  if (!(scale >= -3.0e38f && scale <= 3.0e38f)) return DPTQ_ERR_INVALID_ARG;   // also rejects NaN
  if (T == 0 || B == 0) return DPTQ_OK;
  c.cache.k_pages = const_cast<uint8_t*>(k_pages);
  c.cache.v_pages = const_cast<uint8_t*>(v_pages);
  c.cache.k_scales = const_cast<float*>(k_scales);
  c.cache.v_scales = const_cast<float*>(v_scales);
  c.cache.cu = cu_seqlens;
  c.cache.lengths = lengths;
  c.cache.table = page_table;
  if (!kv8_pointers(c.cache) || !rows_ok(q, ld_q, (int64_t)heads * head_dim)) return DPTQ_ERR_INVALID_ARG;
  if (!out || !lse || !aligned16(out) || !aligned4(lse)) return DPTQ_ERR_INVALID_ARG;
  const int64_t need = dptq::kv8_attention_workspace(c);
  if (need > 0 && (!workspace || !aligned16(workspace) || workspace_bytes < need)) return DPTQ_ERR_INVALID_ARG;
  c.q = q;
  c.ld_q = ld_q;
  c.scale = scale;
  c.out = out;
  c.lse = lse;
  c.workspace = workspace;
  return from_hip(dptq::launch_kv8_attention(c, static_cast<hipStream_t>(stream)));
}

int64_t dptq_token_logprobs_workspace(int64_t M, int64_t V, int32_t top, int32_t dtype) {
  dptq::TokenLogprobs c{};
  if (logprobs_shape(V, M, V, top, dtype, &c) != DPTQ_OK) return -1;
  return M == 0 ? 0 : dptq::token_logprobs_workspace(c);
}

int dptq_token_logprobs(const void* logits, int32_t dtype, int64_t ld, int64_t M, int64_t V,
                        const int64_t* tokens, int32_t top, float* logprobs, float* entropy,
                        float* top_logprobs, int64_t* top_ids, void* workspace, int64_t workspace_bytes,
                        void* stream) {
  dptq::TokenLogprobs c{};
  const int st = logprobs_shape(ld, M, V, top, dtype, &c);
  if (st != DPTQ_OK) return st;
  if (M == 0) return DPTQ_OK;
  if (!logits || !tokens || !logprobs || !entropy || (top > 0 && (!top_logprobs || !top_ids)))
    return DPTQ_ERR_INVALID_ARG;
  const uintptr_t element = c.fp32 ? 4 : 2;
  if (reinterpret_cast<uintptr_t>(logits) % element != 0 || !aligned8(tokens) || !aligned4(logprobs) ||
      !aligned4(entropy) || !aligned4(top_logprobs) || !aligned8(top_ids))
    return DPTQ_ERR_INVALID_ARG;
  const int64_t need = dptq::token_logprobs_workspace(c);
  if (need > 0 && (!workspace || !aligned16(workspace) || workspace_bytes < need)) return DPTQ_ERR_INVALID_ARG;
  c.logits = logits;
  c.tokens = tokens;
  c.logprobs = logprobs;
  c.entropy = entropy;
  c.top_logprobs = top_logprobs;
  c.top_ids = top_ids;
  c.workspace = workspace;
  return from_hip(dptq::launch_token_logprobs(c, static_cast<hipStream_t>(stream)));
}

int64_t dptq_sample_tokens_workspace(int64_t M, int64_t V, int32_t dtype) {
  dptq::SampleTokens c{};
  if (sample_shape(V, M, V, dtype, &c) != DPTQ_OK) return -1;
  return M == 0 ? 0 : dptq::sample_tokens_workspace(c);
}

int dptq_sample_tokens(const void* logits, int32_t dtype, int64_t ld, int64_t M, int64_t V,
                       const float* uniform, const float* temperature, float temperature_all,
                       const int32_t* top_k, int32_t top_k_all, const float* top_p, float top_p_all,
                       const float* min_p, float min_p_all, int64_t* tokens, float* probs,
                       void* workspace, int64_t workspace_bytes, void* stream) {
  dptq::SampleTokens c{};
  const int st = sample_shape(ld, M, V, dtype, &c);
  if (st != DPTQ_OK) return st;
  if (M == 0) return DPTQ_OK;
  if (!logits || !uniform || !tokens || !probs) return DPTQ_ERR_INVALID_ARG;
  const uintptr_t element = c.fp32 ? 4 : 2;
  if (reinterpret_cast<uintptr_t>(logits) % element != 0 || !aligned4(uniform) || !aligned4(temperature) ||
      !aligned4(top_k) || !aligned4(top_p) || !aligned4(min_p) || !aligned8(tokens) || !aligned4(probs))
    return DPTQ_ERR_INVALID_ARG;
  const int64_t need = dptq::sample_tokens_workspace(c);
  if (need > 0 && (!workspace || !aligned16(workspace) || workspace_bytes < need)) return DPTQ_ERR_INVALID_ARG;
  c.logits = logits;
  c.uniform = uniform;
  c.temperature = temperature;
  c.top_k = top_k;
  c.top_p = top_p;
  c.min_p = min_p;
  c.temperature_all = temperature_all;
  c.top_k_all = top_k_all;
  c.top_p_all = top_p_all;
  c.min_p_all = min_p_all;
  c.tokens = tokens;
  c.probs = probs;
  c.workspace = workspace;
  return from_hip(dptq::launch_sample_tokens(c, static_cast<hipStream_t>(stream)));
}

int dptq_layer_policy(int32_t num_layers, const uint8_t* mask, int32_t* bits_out) {
  if (num_layers < 1 || !bits_out) return DPTQ_ERR_INVALID_ARG;
  for (int32_t l = 0; l < num_layers; ++l) {
    bool sensitive;
    if (mask) {
      sensitive = mask[l] != 0;
    } else {
      // Eq. 21: S = {1, 2, 3, L} counted from 1, i.e. {0, 1, 2, L-1}.
      sensitive = l <= 2 || l == num_layers - 1;
    }
    bits_out[l] = sensitive ? 8 : 4;
  }
  return DPTQ_OK;
}

int dptq_prepare_weights(const float* w, int64_t N, int64_t K, int32_t had_size,
                         uint8_t* w_packed, float* w_scales, void* stream) {
  HadSplit hs{};
  int st = check_rotation_shape(N, K, had_size, &hs);
  if (st != DPTQ_OK) return st;
  if (N == 0) return DPTQ_OK;
  if (!w || !w_packed || !w_scales) return DPTQ_ERR_INVALID_ARG;
  if (!aligned16(w) || !aligned16(w_packed) || !aligned16(w_scales)) return DPTQ_ERR_INVALID_ARG;
  return from_hip(dptq::launch_prepare_weights(w, N, (int)K, hs, w_packed, w_scales,
                                               static_cast<hipStream_t>(stream)));
}

}  // extern "C"
