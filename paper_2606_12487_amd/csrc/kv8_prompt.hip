// kv8_attention for many queries a sequence (the formulas: kv8_attention.hip).
//
// A workgroup of four waves takes 128 rows of one KV head of one sequence (row
// r is query token r / group, head r % group: the heads that share a KV head
// share its loads), 32 rows a wave, and walks the pages they see.  Pages come
// into LDS by direct loads, one page ahead; each wave reads the codes from
// there and converts them as it feeds the matrix cores.  Where that makes too
// few workgroups, one takes 64 rows, two waves on every other page each, and
// joins the two halves at the end (KEYS = 2).
//
// The products are those of the decode kernel on 32 x 32 tiles: S^T = K Q^T
// with the K operand's rows in an order that leaves a lane with 16 consecutive
// tokens of each half page, O^T = V^T P^T.
//
// The softmax keeps a reference m instead of the running maximum: weights are
// 2^(s - m), and m moves (with the sums and O rescaled) only where a score
// passes m + 10, then to 4 below it.  A page's v scale goes into the exponent
// as its ratio to the unit U of O, 2^-4 to 2^4; another unit is taken, with O
// rescaled, where the ratio leaves that range.  Weights stay below 2^15, within
// fp16, and are never below their exact size relative to the row's largest:
// the fp16 rounding is the decode kernel's or finer.
//
// Bound by instruction issue: vector instructions (conversions, softmax; 55 % of
// the SIMD cycles) are hardly hidden behind matrix ones (42 %): the two add up.  Prompts
// of 2048 and 1226 queries over 4096 and 3135 keys (64 heads on 8, head size
// 128) take 333 to 349 us, 0.88 to 0.92 PFLOP/s; 1000 queries behind a window of 1024
// (32 heads on 8, head size 64) 25 us.
#include "kv8_attn.h"
#include "lds_load.h"

namespace dptq {
namespace {

// What is fetched ahead for a page beside its codes.
struct Ahead {
  int page;        // of the list place after
  float ks, vs;    // the page's own scales
};
// Waits for the direct loads and for what was fetched with them.
__device__ __forceinline__ void wait_loads(Ahead& x) {
  asm volatile("s_waitcnt vmcnt(0)" : "+v"(x.page), "+v"(x.ks), "+v"(x.vs)::"memory");
}
__device__ __forceinline__ float uniform(float x) {
  return __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(x)));
}
// Waits for the wave's own LDS reads too: a buffer is refilled behind it.
__device__ __forceinline__ void barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// The 16-byte slot of a row, moved so that the 16 lanes of an operand that are
// read together meet 16 different groups of four of the 64 banks.  K rows, token
// t: those lanes hold tokens 4 x + 16 h + y, y < 4, with four different
// (x & 1, h); 256 bytes of banks take 4, 2 or 1 rows.
template <int D>
__device__ __forceinline__ int k_slot(int t, int slot) {
  const int xh = ((t >> 2) & 1) | ((t >> 3) & 2);
  return slot ^ (D == 64 ? xh : D == 128 ? ((t >> 1) & 1) | xh << 1 : (t & 3) | xh << 2);
}
// V rows, channel d: 64 bytes, four to a line of banks.
__device__ __forceinline__ int v_slot(int d, int slot) { return slot ^ ((d >> 2) & 3); }

template <int D, int KEYS>
__global__ void __launch_bounds__(256, D == 256 ? 1 : 2) kv8_prompt_kernel(AttnArgs a) {
  constexpr int kThreads = 256 / KEYS, kRows = 128 / KEYS;   // of the waves that share pages
  constexpr int kC = D / 32;                       // 32-channel parts of a row
  constexpr int kBytes = kPage * D;                // codes of a page and head
  constexpr int kLoads = kBytes / 16 / kThreads;   // 16-byte loads of a thread for K, and for V
  extern __shared__ uint8_t all_lds[];
  const int keys = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kThreads);   // which of the pages
  const int tid = threadIdx.x % kThreads, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const uint32_t lds_at = (uint32_t)keys * 4 * kBytes;
  uint8_t* const lds = all_lds + lds_at;           // two buffers of K, two of V
  const int col = lane & 31, hh = lane >> 5;
  const int head = (int)blockIdx.x, b = (int)blockIdx.z / a.splits, part = (int)blockIdx.z % a.splits;
  const KvSeq seq = kv_seq(a.cu, a.lengths, b, a.T);
  const int rows = seq.count * a.group;   // T * heads < 2^30
  const int tiles = (rows + kRows - 1) / kRows;
  const int32_t* const table = a.table + (int64_t)b * a.max_pages;
  const float sign = a.scale_log2 < 0.0f ? -1.0f : 1.0f;

  // Where this thread's 16-byte loads of a page come from: slot s of LDS, in
  // order, takes the row's slot that is moved there.
  uint32_t from_k[kLoads], from_v[kLoads];
#pragma unroll
  for (int i = 0; i < kLoads; ++i) {
    const int s = i * kThreads + tid;
    const int t = s / (D / 16), ks = s % (D / 16), d = s / 4, vs = s % 4;
    from_k[i] = (uint32_t)(t * D + 16 * k_slot<D>(t, ks));
    from_v[i] = (uint32_t)(d * kPage + 16 * v_slot(d, vs));
  }

  // Tiles from the sequence's end: those that see most come first.
  for (int tile = tiles - 1 - (int)blockIdx.y; tile >= 0; tile -= (int)gridDim.y) {
    const int row0 = tile * kRows;
    const int last_row = min(row0 + kRows, rows) - 1;
    const int wrow0 = min(row0 + 32 * wave, last_row), wrow1 = min(row0 + 32 * wave + 31, last_row);
    const int row = min(row0 + 32 * wave + col, last_row);   // lanes past the end repeat the last row
    const int token = row / a.group, g = row % a.group;
    const int pos = seq.start + token;
    const int wmin = __builtin_amdgcn_readfirstlane(seq.start + wrow0 / a.group);
    const int wmax = __builtin_amdgcn_readfirstlane(seq.start + wrow1 / a.group);
    const Visible vis = visible_pages(seq.start + row0 / a.group, seq.start + last_row / a.group, a.window, a.sinks,
                                      a.max_pages);
    const int begin = min(part * a.chunk, vis.total);
    const int end = part == a.splits - 1 ? vis.total : min(begin + a.chunk, vis.total);

    // Queries: chunk (C, e) gives lane (col, hh) channels 32 C + 16 hh + 8 e and up.
    half8 qf[kC][2];
    const __half* const qrow = a.q + (int64_t)(seq.first_row + token) * a.ld_q + (int64_t)(head * a.group + g) * D;
#pragma unroll
    for (int C = 0; C < kC; ++C)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        qf[C][e] = *reinterpret_cast<const half8*>(qrow + 32 * C + 16 * hh + 8 * e);
        qf[C][e] *= (_Float16)sign;
      }

    float16v o[D / 32];
#pragma unroll
    for (int t = 0; t < D / 32; ++t)
#pragma unroll
      for (int e = 0; e < 16; ++e) o[t][e] = 0.0f;
    float m = -INFINITY, l = 0.0f, unit = 0.0f, inv_unit = 0.0f;   // unit 0: none yet

    // Pages that are not there are passed over.
    const auto there = [&](int page) { return (uint32_t)page < (uint32_t)a.num_pages; };
    const auto entry = [&](int i) { return i < end ? table[vis.page(i)] : -1; };
    const auto load_k = [&](int page, int buf) {
      const uint8_t* const from = a.k_pages + ((int64_t)page * a.kv_heads + head) * kBytes;
#pragma unroll
      for (int n = 0; n < kLoads; ++n)
        load_lds16(from, from_k[n], lds_at + (uint32_t)(buf * kBytes + wave * 1024 + n * 16 * kThreads));
    };
    const auto load_v = [&](int page, int buf) {
      const uint8_t* const from = a.v_pages + ((int64_t)page * a.kv_heads + head) * kBytes;
#pragma unroll
      for (int n = 0; n < kLoads; ++n)
        load_lds16(from, from_v[n], lds_at + (uint32_t)((2 + buf) * kBytes + wave * 1024 + n * 16 * kThreads));
    };
    // S^T of half page u from a K buffer: row 8 x + 4 h + y of the operand is
    // token 32 u + 16 h + 4 x + y.
    const int ktok = 16 * ((col >> 2) & 1) + 4 * (col >> 3) + (col & 3);
    const auto scores = [&](int buf, int u) {
      const int t = 32 * u + ktok;
      const uint8_t* const kb = lds + buf * kBytes + t * D;
      float16v s;
#pragma unroll
      for (int e = 0; e < 16; ++e) s[e] = 0.0f;
#pragma unroll
      for (int C = 0; C < kC; ++C) {
        const uint4 kc = *reinterpret_cast<const uint4*>(kb + 16 * k_slot<D>(t, 2 * C + hh));
        s = __builtin_amdgcn_mfma_f32_32x32x16_f16(codes8(kc.x, kc.y), qf[C][0], s, 0, 0, 0);
        s = __builtin_amdgcn_mfma_f32_32x32x16_f16(codes8(kc.z, kc.w), qf[C][1], s, 0, 0, 0);
      }
      return s;
    };

    // The scores of the next page are formed while a page goes through the
    // softmax and the second product; K of the one after and V of the next come
    // in meanwhile, with their scales and the table's entry after them.
    const int first = begin + keys;
    int page = __builtin_amdgcn_readfirstlane(entry(first));           // of place i
    int page1 = __builtin_amdgcn_readfirstlane(entry(first + KEYS));   // the next
    Ahead ahead{entry(first + 2 * KEYS), 0.0f, 0.0f};                  // the one after; scales of place i
    float16v s0, s1;
#pragma unroll
    for (int e = 0; e < 16; ++e) s0[e] = s1[e] = 0.0f;
    if (begin < end) {
      if (there(page)) {
        load_k(page, 0);
        load_v(page, 0);
        ahead.ks = a.k_scales[(int64_t)page * a.kv_heads + head];
        ahead.vs = a.v_scales[(int64_t)page * a.kv_heads + head];
      }
      if (there(page1)) load_k(page1, 1);
      wait_loads(ahead);
      barrier();
      if (there(page)) {
        s0 = scores(0, 0);
        s1 = scores(0, 1);
      }
    }
    for (int turn = begin, buf = 0; turn < end; turn += KEYS, buf ^= 1) {
      const int i = turn + keys, j0 = vis.page(i) * kPage;   // past the end: no page
      if (turn > begin) wait_loads(ahead);
      const float ks = uniform(ahead.ks), vs = uniform(ahead.vs);
      const int page2 = __builtin_amdgcn_readfirstlane(ahead.page);
      barrier();   // everyone's loads are in, and everyone is done with the buffers of the last turn
      ahead.page = entry(i + 3 * KEYS);
      if (there(page1)) {
        load_v(page1, buf ^ 1);
        ahead.ks = a.k_scales[(int64_t)page1 * a.kv_heads + head];
        ahead.vs = a.v_scales[(int64_t)page1 * a.kv_heads + head];
      }
      if (there(page2)) load_k(page2, buf);
      const bool here = there(page);
      uint8_t* const vb = lds + (2 + buf) * kBytes;
      // V's slots past the sequence's end may hold anything: they are cleared,
      // so that no NaN of theirs meets the zero weight.
      if (vis.page(min(turn + KEYS, end) - 1) * kPage + kPage > seq.length) {   // the same for every wave
#pragma unroll
        for (int n = 0; n < kLoads; ++n) {
          const int slot = n * kThreads + tid, d = slot / 4;
          const int held = seq.length - j0 - 16 * v_slot(d, slot % 4);
          uint4* const w = reinterpret_cast<uint4*>(vb + 16 * slot);
          *w = make_uint4(w->x & held_mask(held, 0), w->y & held_mask(held, 4), w->z & held_mask(held, 8),
                          w->w & held_mask(held, 12));
        }
        barrier();
      }
      if (here && page_any(j0, wmin, wmax, a.window, a.sinks)) {
        if (!page_whole(j0, wmin, wmax, a.window, a.sinks)) {
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            s0[e] = sees(pos, j0 + 16 * hh + e, a.window, a.sinks) ? s0[e] : -INFINITY;
            s1[e] = sees(pos, j0 + 32 + 16 * hh + e, a.window, a.sinks) ? s1[e] : -INFINITY;
          }
        }
        // c > 0 also where the scale is 0: -inf stays -inf.
        const float c = fmaxf(fabsf(a.scale_log2) * ks, 1e-37f);
        float top = fmaxf(s0[0], s1[0]);
#pragma unroll
        for (int e = 1; e < 16; ++e) top = fmaxf(fmaxf(top, s0[e]), s1[e]);
        top *= c;
        float ratio = vs * inv_unit;
        const bool other_unit = !(ratio >= 0.0625f && ratio <= 16.0f);
        if (__any(top > m + 10.0f) || other_unit) {
          // Both lanes of a row (halves of the tokens) move its reference alike.
          const float row_top = fmaxf(top, __shfl_xor(top, 32));
          const bool up = row_top > m + 10.0f;
          const float m_new = up ? row_top - 4.0f : m;
          const float alpha = m == -INFINITY ? 0.0f : exp2_hw(m - m_new);
          float fix = alpha;
          if (other_unit) {
            const float inv = __builtin_amdgcn_rcpf(vs);
            fix = alpha * (unit * inv);
            unit = vs;
            inv_unit = inv;
            ratio = 1.0f;
          }
          m = m_new;
          l *= alpha;
#pragma unroll
          for (int t = 0; t < D / 32; ++t) o[t] *= fix;
        }
        // Weights with the v scale in them; their sum without it.
        const float base = m == -INFINITY ? 0.0f : m;
        const float shift = __builtin_amdgcn_logf(ratio) - base;
        // (Scores of a page that is not there are never used.)
        const float16v n0 = scores(buf ^ 1, 0), n1 = scores(buf ^ 1, 1);
        float sum = 0.0f;
        half8 p[2][2];
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const float x = exp2_hw(fmaf(s0[e], c, shift)), y = exp2_hw(fmaf(s1[e], c, shift));
          sum += x;
          sum += y;
          p[0][e / 8][e % 8] = (_Float16)x;
          p[1][e / 8][e % 8] = (_Float16)y;
        }
        l = fmaf(sum, __builtin_amdgcn_rcpf(ratio), l);
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int t = 0; t < D / 32; ++t) {
            const int d = 32 * t + col;
            const uint4 vc = *reinterpret_cast<const uint4*>(vb + d * kPage + 16 * v_slot(d, 2 * u + hh));
            o[t] = __builtin_amdgcn_mfma_f32_32x32x16_f16(codes8(vc.x, vc.y), p[u][0], o[t], 0, 0, 0);
            o[t] = __builtin_amdgcn_mfma_f32_32x32x16_f16(codes8(vc.z, vc.w), p[u][1], o[t], 0, 0, 0);
          }
        s0 = n0;
        s1 = n1;
      } else {
        s0 = scores(buf ^ 1, 0);
        s1 = scores(buf ^ 1, 1);
      }
      page = page1;
      page1 = page2;
    }
    l += __shfl_xor(l, 32);

    if constexpr (KEYS == 2) {
      // The two halves' sums, relative to the larger reference, in units of 1.
      float* const o_of = reinterpret_cast<float*>(all_lds);
      float* const ml_of = o_of + 16 * (D / 32) * kThreads;
      barrier();   // the pages are done with
      if (keys == 1) {
#pragma unroll
        for (int t = 0; t < D / 32; ++t)
#pragma unroll
          for (int e = 0; e < 16; ++e) o_of[(16 * t + e) * kThreads + tid] = o[t][e] * unit;
        ml_of[tid] = m;
        ml_of[kThreads + tid] = l;
      }
      barrier();
      if (keys == 0) {
        const float m1 = ml_of[tid], both = fmaxf(m, m1), ref = both == -INFINITY ? 0.0f : both;
        const float f0 = exp2_hw(m - ref), f1 = exp2_hw(m1 - ref);
#pragma unroll
        for (int t = 0; t < D / 32; ++t)
#pragma unroll
          for (int e = 0; e < 16; ++e)
            o[t][e] = o[t][e] * (f0 * unit) + f1 * o_of[(16 * t + e) * kThreads + tid];
        l = f0 * l + f1 * ml_of[kThreads + tid];
        m = both;
        unit = 1.0f;
      }
    }

    if (keys == 0 && row0 + 32 * wave + col < rows) {
      const int64_t to = ((int64_t)seq.first_row + token) * a.heads + head * a.group + g;
      if (a.splits == 1) {
        const float f = l > 0.0f ? unit / l : l;   // 0: nothing seen; NaN stays
#pragma unroll
        for (int t = 0; t < D / 32; ++t)
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            __half2 h[2];
            h[0] = __floats2half2_rn(o[t][4 * x] * f, o[t][4 * x + 1] * f);
            h[1] = __floats2half2_rn(o[t][4 * x + 2] * f, o[t][4 * x + 3] * f);
            *reinterpret_cast<uint2*>(a.out + to * D + 32 * t + 8 * x + 4 * hh) = *reinterpret_cast<const uint2*>(h);
          }
        if (hh == 0) a.lse[to] = m * kLn2 + logf(l);
      } else {
        const int64_t slot = (int64_t)part * a.T * a.heads + to;
        if (begin < end) {   // parts without pages come last
#pragma unroll
          for (int t = 0; t < D / 32; ++t)
#pragma unroll
            for (int x = 0; x < 4; ++x)
              *reinterpret_cast<float4v*>(a.part_o + slot * D + 32 * t + 8 * x + 4 * hh) =
                  float4v{o[t][4 * x], o[t][4 * x + 1], o[t][4 * x + 2], o[t][4 * x + 3]} * unit;
        }
        if (hh == 0) a.part_ml[slot] = make_float2(m, l);
      }
    }
    barrier();   // the buffers are free for the next tile
  }
}

template <int D, int KEYS>
hipError_t launch(const AttnArgs& a, int64_t B, int64_t max_q, hipStream_t stream) {
  constexpr int kPages = KEYS * 4 * kPage * D, kJoin = (16 * (D / 32) + 2) * 4 * (256 / KEYS);
  constexpr int kLds = KEYS == 2 && kJoin > kPages ? kJoin : kPages, kRows = 128 / KEYS;
  const int64_t tiles = (max_q * a.group + kRows - 1) / kRows;
  // The heads first: with 8 of them a head's pages stay in one XCD's L2.  Then a
  // sequence's tiles: workgroups go to the shader engines in turn, and an order
  // that alternates long and short sequences gives all long ones to the same
  // engines (391 against 356 us for two sequences of 2048 and 1226 queries).
  const dim3 grid((unsigned)a.kv_heads, (unsigned)(tiles < 65535 ? tiles : 65535), (unsigned)(B * a.splits));
  if constexpr (kLds > 65536) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kv8_prompt_kernel<D, KEYS>),
                                             hipFuncAttributeMaxDynamicSharedMemorySize, kLds);
    if (e != hipSuccess) return e;
  }
  kv8_prompt_kernel<D, KEYS><<<grid, 256, kLds, stream>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_kv8_prompt(const AttnArgs& a, int head_dim, int rows, int64_t B, int64_t max_q,
                             hipStream_t stream) {
  switch (head_dim) {
    case 64: return rows == 128 ? launch<64, 1>(a, B, max_q, stream) : launch<64, 2>(a, B, max_q, stream);
    case 128: return rows == 128 ? launch<128, 1>(a, B, max_q, stream) : launch<128, 2>(a, B, max_q, stream);
    case 256: return rows == 128 ? launch<256, 1>(a, B, max_q, stream) : launch<256, 2>(a, B, max_q, stream);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace dptq
