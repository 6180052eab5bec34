// Norms of queries and keys per head, their rotation, and the store of keys and
// values into the cache, in one pass over the fused projection
// (fsched_qk_norm_rope).
//
//   y = x / sqrt(mean(x^2) + eps) * w;  (a, b) -> (a cos - b sin, b cos + a sin)
//
// Bound by memory: each element is read and written once, with a few operations
// in between.  A head vector lies across head_dim / 8 lanes, 16 bytes each (one
// load, one store); its mean is a butterfly over those lanes, and with pairs
// (i, i + rot/2) the partner's elements come from the lane rot/16 away.  The
// lanes' cosines and sines (64 bytes against 16 of x) are loaded once per token
// and kept for all the heads that the wave takes of it.
// Measured: 32,771 tokens of 48 heads of 128 (f16), 163 us or 5.0 TB/s, a large copy's
// rate; 64 tokens, 3.7 us.
#include <hip/hip_runtime.h>

#include "half.hpp"
#include "step_common.hpp"

namespace fs {
namespace {

constexpr int THREADS = 256;

template <class T, int D, bool INTER>
__global__ __launch_bounds__(THREADS) void qk_rope_kernel(RopeArgs a, int chunks, int per_chunk) {
  constexpr int LANES = D / 8;        // lanes of one head vector
  constexpr int HEADS = 64 / LANES;   // head vectors a wave holds at once
  using x8 = typename T::x8;
  using elem = typename T::elem;
  const int lane = threadIdx.x & 63;
  const int sub = lane & (LANES - 1), grp = lane / LANES;
  const int64_t w = (int64_t)blockIdx.x * (THREADS / 64) + (threadIdx.x >> 6);
  const int64_t t = w / chunks;
  if (t >= a.n_tok) return;
  const int heads = a.q_heads + 2 * a.kv.kv_heads;
  const int h0 = (int)(w % chunks) * per_chunk, h1 = min(heads, h0 + per_chunk);

  const int d0 = sub * 8, half = a.rot_dim >> 1;
  const bool rotated = d0 < a.rot_dim;
  bool known = true;  // the token has a row of the rotation table
  float c[8], s[8];
  if (a.rot_dim > 0) {
    const int pos = a.positions[t];
    known = pos >= 0 && pos < a.n_pos;
    if (known && rotated) {
      const float* row = a.cos_sin + (int64_t)pos * a.rot_dim;
      if (INTER) {
        const f32x4 x = *(const f32x4*)(row + d0 / 2);
        const float* sn = row + half + d0 / 2;
        const f32x4 y = *(const f32x4*)sn;
#pragma unroll
        for (int i = 0; i < 4; ++i) c[i] = x[i], s[i] = y[i];
      } else {
        const int at = d0 < half ? d0 : d0 - half;
#pragma unroll
        for (int i = 0; i < 8; i += 4) {
          const f32x4 x = *(const f32x4*)(row + at + i);
          const f32x4 y = *(const f32x4*)(row + half + at + i);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            c[i + j] = x[j];
            s[i + j] = d0 < half ? -y[j] : y[j];
          }
        }
      }
    }
  }
  // where the token's keys and values go: a slot of the cache, or nowhere
  const int slot = a.slots ? a.slots[t] : -1;
  const int page = slot >> a.kv.page_shift;
  const int off = slot & ((1 << a.kv.page_shift) - 1);
  const bool store = slot >= 0 && page < a.kv.n_pages && known;
  const int partner = lane + (d0 < half ? half / 8 : -(half / 8));

  const elem* in = (const elem*)a.qkv + t * a.qkv_stride + d0;
  for (int h = h0 + grp; h - grp < h1; h += HEADS) {
    const bool on = h < h1;  // lanes past the last head help their wave's exchanges
    x8 raw = {};
    if (on) raw = __builtin_nontemporal_load((const x8*)(in + (int64_t)h * D));
    const bool is_q = h < a.q_heads, is_k = !is_q && h < a.q_heads + a.kv.kv_heads;
    float x[8];
    float sq = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      x[i] = (float)raw[i];
      sq = fmaf(x[i], x[i], sq);
    }
    const void* weight = is_q ? a.q_weight : is_k ? a.k_weight : nullptr;
#pragma unroll
    for (int d = 1; d < LANES; d <<= 1) sq += __shfl_xor(sq, d);
    if (weight) {
      const float r = 1.0f / sqrtf(sq * (1.0f / D) + a.eps);
      const x8 g = *(const x8*)((const elem*)weight + d0);
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = x[i] * r * (float)g[i];
    }
    if (a.rot_dim > 0) {
      if (INTER) {
        if (rotated && known && (is_q || is_k)) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float p = x[2 * i], q = x[2 * i + 1];
            x[2 * i] = p * c[i] - q * s[i];
            x[2 * i + 1] = q * c[i] + p * s[i];
          }
        }
      } else {
        float y[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = __shfl(x[i], partner & 63);
        if (rotated && known && (is_q || is_k)) {
#pragma unroll
          for (int i = 0; i < 8; ++i) x[i] = x[i] * c[i] + y[i] * s[i];
        }
      }
    }
    if (!on) continue;
    x8 res;
#pragma unroll
    for (int i = 0; i < 8; ++i) res[i] = (elem)x[i];
    if (is_q) {
      const x8 zero = {};
      *(x8*)((elem*)a.q_out + t * a.q_token + (int64_t)h * a.q_head + d0) = known ? res : zero;
    } else if (store) {
      const int64_t kh = h - a.q_heads - (is_k ? 0 : a.kv.kv_heads);
      const int64_t at = is_k ? page * a.kv.k_page + kh * a.kv.k_head + off * a.kv.k_slot
                              : page * a.kv.v_page + kh * a.kv.v_head + off * a.kv.v_slot;
      elem* base = (elem*)(is_k ? a.kv.k : a.kv.v);
      *(x8*)(base + at + d0) = is_k ? res : raw;
    }
  }
}

template <class T, int D>
hipError_t launch(const RopeArgs& a, int n_cu, hipStream_t s) {
  const int heads = a.q_heads + 2 * a.kv.kv_heads, at_once = 64 / (D / 8);
  // All heads of a token in one wave (its rotation row is loaded once), unless
  // that leaves the device short of waves: then as few heads as a wave holds (64 tokens,
  // traced: 4.0 us where 2 waves per unit are enough, 3.2 with 8, 3.4 with 32).
  int chunks = 1;
  const int most = (heads + at_once - 1) / at_once;
  while (chunks < most && (int64_t)a.n_tok * chunks < 8 * (int64_t)n_cu) chunks *= 2;
  if (chunks > most) chunks = most;
  int per = (heads + chunks - 1) / chunks;
  per = (per + at_once - 1) / at_once * at_once;
  chunks = (heads + per - 1) / per;
  const int64_t waves = (int64_t)a.n_tok * chunks;
  const dim3 grid((unsigned)((waves + THREADS / 64 - 1) / (THREADS / 64))), block(THREADS);
  if (a.interleaved) qk_rope_kernel<T, D, true><<<grid, block, 0, s>>>(a, chunks, per);
  else qk_rope_kernel<T, D, false><<<grid, block, 0, s>>>(a, chunks, per);
  return hipGetLastError();
}

template <class T>
hipError_t launch_dim(const RopeArgs& a, int head_dim, int n_cu, hipStream_t s) {
  switch (head_dim) {
    case 64: return launch<T, 64>(a, n_cu, s);
    case 128: return launch<T, 128>(a, n_cu, s);
    default: return launch<T, 256>(a, n_cu, s);
  }
}

}  // namespace

hipError_t launch_qk_rope(const RopeArgs& a, int dtype, int head_dim, int n_cu, hipStream_t s) {
  return dtype == FSCHED_BF16 ? launch_dim<Bf16>(a, head_dim, n_cu, s)
                              : launch_dim<F16>(a, head_dim, n_cu, s);
}

}  // namespace fs
