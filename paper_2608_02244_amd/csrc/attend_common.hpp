// Parts shared by the attention kernels (attend_rows.hpp, attend_tiles.hpp,
// attend.hip).
//
// Every kernel keeps, per row (a token and query head), the running maximum m of
// its scores in base 2, the sum l of 2^(s - m) and the unnormalised output o.
// Parts over disjoint keys join by  m = max m_i,  l = sum l_i 2^(m_i - m),
// o = sum o_i 2^(m_i - m);  the result is o / l and lse = (m + log2 l) ln 2.
//
// Scores, m, l and o are 32-bit.  The weights 2^(s - m) are rounded to the values' type for
// the second product, whose operands the matrix unit takes in 16 bits; l sums them before
// that, so lse keeps its 32 bits.  Relative distance of the outputs from 64 bits: 2.2e-3 in
// bf16 and 2.7e-4 in f16, against 1.7e-3 and 2.1e-4 where only the result is rounded.  A
// second product with the weights' remainders would take that back for half as many
// products again.
#pragma once
#include <hip/hip_runtime.h>

#include "half.hpp"
#include "step_common.hpp"

namespace fs {

constexpr int ATT_THREADS = 256, ATT_WAVES = ATT_THREADS / 64;
// The kernels' WIDE forms are for pages of 2^4 tokens and more.  With and without them:
// prompts 672 / 718 us a call, chunks beside decoding requests 109 / 111; decode alike (64
// requests 55.6 / 55.1).
constexpr int WIDE_SHIFT = 4;
constexpr float NEG_INF = -__builtin_inff();
constexpr float LN2 = 0.6931471805599453f;

// A request's rows and tokens, from device data that is checked here: nothing
// that the kernels index with leaves its array, whatever q_start and kv_len hold.
struct Request {
  int q0, q_len;  // its rows of q; tokens past max_q count but are not computed
  int kv;         // own tokens held
};

__device__ __forceinline__ Request request_of(const AttnArgs& a, int r) {
  Request x;
  const int b = a.q_start[r], e = a.q_start[r + 1];
  x.q0 = min(max(0, b), a.n_tok);
  x.q_len = min(max(e, x.q0), a.n_tok) - x.q0;
  x.kv = min(max(0, a.kv_len[r]), a.width << a.kv.page_shift);
  return x;
}

// Own keys (counted from the end of the prefix) that some row of a set of tokens
// sees, as blocks of BLOCK keys: the first `sink_blocks`, then those from
// `first_block` on; `blocks` in all.
struct Span {
  int sink_blocks, first_block, blocks;
  __device__ __forceinline__ int block(int i) const {
    return i < sink_blocks ? i : first_block + (i - sink_blocks);
  }
};

// Tokens at own indices p0 .. p1 (position minus prefix; may be negative) over
// keys 0 .. n-1.  `offset`: position of key 0 (the prefix's length, or 0 for the
// prefix itself, whose tokens all come later).
template <int BLOCK>
__device__ __forceinline__ Span span_of(int p0, int p1, int n, int window, int n_sink,
                                        int offset) {
  Span s;
  const int hi = min(n, p1 + 1);  // keys past p1 are seen by none
  int lo = 0, sinks = 0;
  if (window > 0) {
    lo = max(0, p0 - window + 1);
    sinks = min(max(0, n_sink - offset), hi);
  }
  const int end = hi > 0 ? (hi + BLOCK - 1) / BLOCK : 0;
  s.first_block = min(lo / BLOCK, end);
  s.sink_blocks = (sinks + BLOCK - 1) / BLOCK;
  if (s.sink_blocks >= s.first_block) s.sink_blocks = s.first_block;  // no gap between them
  s.blocks = s.sink_blocks + (end - s.first_block);
  return s;
}

__device__ __forceinline__ int uni_int(int v) { return __builtin_amdgcn_readfirstlane(v); }

// Largest and summed value over the lanes that hold parts of one row: lanes
// equal mod 32 (xor 32), or mod 16 (xor 16 and 32).
__device__ __forceinline__ float max_xor32(float x) {
  const u32x2 r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, x),
                                                   __builtin_bit_cast(uint32_t, x), false, false);
  return fmaxf(__builtin_bit_cast(float, (uint32_t)r[0]),
               __builtin_bit_cast(float, (uint32_t)r[1]));
}
__device__ __forceinline__ float max_xor16(float x) {
  const u32x2 r = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(uint32_t, x),
                                                   __builtin_bit_cast(uint32_t, x), false, false);
  return fmaxf(__builtin_bit_cast(float, (uint32_t)r[0]),
               __builtin_bit_cast(float, (uint32_t)r[1]));
}
__device__ __forceinline__ float sum_xor32(float x) {
  const u32x2 r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, x),
                                                   __builtin_bit_cast(uint32_t, x), false, false);
  return __builtin_bit_cast(float, (uint32_t)r[0]) + __builtin_bit_cast(float, (uint32_t)r[1]);
}
__device__ __forceinline__ float sum_xor16(float x) {
  const u32x2 r = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(uint32_t, x),
                                                   __builtin_bit_cast(uint32_t, x), false, false);
  return __builtin_bit_cast(float, (uint32_t)r[0]) + __builtin_bit_cast(float, (uint32_t)r[1]);
}

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// What a score's exponential is taken against (mu): the running maximum less BIAS,
// moved only when a score would exceed it by TAU more.  P is then at most
// 2^(BIAS + TAU), within f16; small weights keep their bits in f16, whose
// smallest normal number is 2^-14 (bf16 needs no bias), and the outputs are
// rescaled a few times per row rather than at every new maximum.
template <class T>
constexpr float BIAS = __is_same(T, F16) ? 8.0f : 0.0f;
constexpr float TAU = 6.0f;

// 2^(x - m) where m may be -infinity (no key so far): then 0.
__device__ __forceinline__ float part_scale(float x, float m) {
  return x == NEG_INF ? 0.0f : exp2_fast(x - m);
}

}  // namespace fs
