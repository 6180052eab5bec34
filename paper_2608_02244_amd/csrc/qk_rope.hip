// Norms of queries and keys per head, their rotation, and the store of keys and
// values into the cache, in one pass over the fused projection
// (fsched_qk_norm_rope), of 16 bits or of 4 (fsched_qk_norm_rope4), and the read back of
// the latter (fsched_kv4_read).
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
//
// Into a cache of 4 bits, keys are normed and rotated in 64 bits, so that their codes are
// those of the numbers themselves and not of one order of summing them: a number next to
// the border of two codes is off by a third of itself on the other side.  Bound by these
// instructions beside the bytes: 32,771 tokens of 48 heads of 128 (f16), 174 us for the
// store (72 % of the vector issue; 186 with the norm of keys and values taken in 32 bits too)
// and 42 for reading them back, 5.2 TB/s; 64 tokens, 4.8 and 2.8 us.
#include <hip/hip_runtime.h>

#include "fp4.hpp"
#include "step_common.hpp"

namespace fs {
namespace {

constexpr int THREADS = 256;

// 1 / sqrt(s) in 64 bits: two steps of Newton's from the 32-bit one (2^-22, then 2^-43, then
// 2^-53), where 32 bits have room for s.
__device__ __forceinline__ double inverse_root(double s) {
  if (!(s > 1e-30 && s < 1e30)) return 1.0 / sqrt(s);
  double r = (double)__builtin_amdgcn_rsqf((float)s);
#pragma unroll
  for (int i = 0; i < 2; ++i) r = r * fma(-0.5 * s * r, r, 1.5);
  return r;
}

// A key in 64 bits: normed (weight given) and rotated (c, s given) as the kernel below does.
template <class T, int D, bool INTER>
__device__ __forceinline__ void exact_key(typename T::x8 raw, const void* weight, float eps,
                                          bool turns, bool rotated, const float* c,
                                          const float* s, int d0, int partner, float* out) {
  using x8 = typename T::x8;
  using elem = typename T::elem;
  double x[8], sq = 0.0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    x[i] = (double)(float)raw[i];
    sq = fma(x[i], x[i], sq);
  }
  if (weight) {
#pragma unroll
    for (int d = 1; d < D / 8; d <<= 1) sq += __shfl_xor(sq, d);
    const double r = inverse_root(sq * (1.0 / D) + (double)eps);
    const x8 g = *(const x8*)((const elem*)weight + d0);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = x[i] * r * (double)(float)g[i];
  }
  if (turns) {
    if (INTER) {
      if (rotated) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const double p = x[2 * i], q = x[2 * i + 1];
          x[2 * i] = p * (double)c[i] - q * (double)s[i];
          x[2 * i + 1] = q * (double)c[i] + p * (double)s[i];
        }
      }
    } else {
      double y[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = __shfl(x[i], partner & 63);
      if (rotated) {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = x[i] * (double)c[i] + y[i] * (double)s[i];
      }
    }
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) out[i] = to_odd(x[i]);
}

// FP4: the cache holds 4 bits an element; its strides are bytes, k_slot that of a group.
// Six blocks per compute unit then (80 registers): stored and read back, the case above
// 202 us with 6, 214 with 5, 207 with 8.
template <class T, int D, bool INTER, bool FP4>
__global__ __launch_bounds__(THREADS, FP4 ? 6 : 1) void qk_rope_kernel(RopeArgs a, int chunks,
                                                                      int per_chunk) {
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
  x8 next = {};
  auto head_at = [&](int h) {
    return __builtin_nontemporal_load((const x8*)(in + (int64_t)h * D));
  };
  if (FP4 && h0 + grp < h1) next = head_at(h0 + grp);
  for (int h = h0 + grp; h - grp < h1; h += HEADS) {
    const bool on = h < h1;  // lanes past the last head help their wave's exchanges
    x8 raw = {};
    if constexpr (FP4) {  // the heads' work is uneven, so the next ones are under way
      raw = next;
      if (h + HEADS < h1) next = head_at(h + HEADS);
    } else {
      if (on) raw = head_at(h);
    }
    const bool is_q = h < a.q_heads, is_k = !is_q && h < a.q_heads + a.kv.kv_heads;
    float x[8];
    const void* weight = is_q ? a.q_weight : is_k ? a.k_weight : nullptr;
    // keys and values of a cache of 4 bits: below
    const bool here = !FP4 || __ballot(is_q) != 0;
    float sq = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      x[i] = (float)raw[i];
      sq = fmaf(x[i], x[i], sq);
    }
    if (here) {
#pragma unroll
      for (int d = 1; d < LANES; d <<= 1) sq += __shfl_xor(sq, d);
    }
    if (here && weight) {
      const float r = 1.0f / sqrtf(sq * (1.0f / D) + a.eps);
      const x8 g = *(const x8*)((const elem*)weight + d0);
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = x[i] * r * (float)g[i];
    }
    if (here && a.rot_dim > 0) {
      if (INTER) {
        if (rotated && known && (is_q || is_k)) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float p = x[2 * i], q = x[2 * i + 1];
            if constexpr (FP4) {  // rounded as the compiler's choice for the other is
              x[2 * i] = fmaf(p, c[i], -(q * s[i]));
              x[2 * i + 1] = fmaf(p, s[i], q * c[i]);
            } else {
              x[2 * i] = p * c[i] - q * s[i];
              x[2 * i + 1] = q * c[i] + p * s[i];
            }
          }
        }
      } else {
        float y[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = __shfl(x[i], partner & 63);
        if (rotated && known && (is_q || is_k)) {
#pragma unroll
          for (int i = 0; i < 8; ++i)
            x[i] = FP4 ? fmaf(x[i], c[i], y[i] * s[i]) : x[i] * c[i] + y[i] * s[i];
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
    } else if constexpr (FP4) {
      if (!store) continue;  // a head's lanes alike
      using G = Group4<D>;
      float y[8];
      if (is_k) {
        exact_key<T, D, INTER>(raw, weight, a.eps, a.rot_dim > 0, rotated, c, s, d0, partner, y);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = (float)raw[i];
      }
      uint32_t top = 0;  // as whole numbers, in which NaN and infinity are above all others
#pragma unroll
      for (int i = 0; i < 8; ++i)
        top = max(top, __builtin_bit_cast(uint32_t, y[i]) & 0x7fffffffu);
      top = max(top, (uint32_t)__shfl_xor((int)top, 1));
      top = max(top, (uint32_t)__shfl_xor((int)top, 2));
      const int byte = scale_byte<T>(top);
      const uint32_t code = byte == 255 ? 0 : codes8(y, scale_of(byte));
      const int64_t kh = h - a.q_heads - (is_k ? 0 : a.kv.kv_heads);
      char* group = (char*)const_cast<void*>(a.kv.k) + page * a.kv.k_page + kh * a.kv.k_head +
                    (off >> GROUP_SHIFT) * a.kv.k_slot;
      const int tok = off & (GROUP - 1);
      if (is_k) {
        *(uint32_t*)(group + G::key(tok) + sub * 4) = code;
      } else if constexpr (D == 64) {  // two pieces of 4 elements
        *(uint16_t*)(group + G::value(tok, 2 * sub)) = (uint16_t)code;
        *(uint16_t*)(group + G::value(tok, 2 * sub + 1)) = (uint16_t)(code >> 16);
      } else {
        constexpr int PER = D / 128;  // lanes of a piece
        *(uint32_t*)(group + G::value(tok, sub / PER) + sub % PER * 4) = code;
      }
      if ((sub & 3) == 0)
        *(uint8_t*)(group + (is_k ? G::key_scale(tok, sub >> 2) : G::value_scale(tok, sub >> 2))) =
            (uint8_t)byte;
    } else if (store) {
      const int64_t kh = h - a.q_heads - (is_k ? 0 : a.kv.kv_heads);
      const int64_t at = is_k ? page * a.kv.k_page + kh * a.kv.k_head + off * a.kv.k_slot
                              : page * a.kv.v_page + kh * a.kv.v_head + off * a.kv.v_slot;
      elem* base = (elem*)(is_k ? a.kv.k : a.kv.v);
      *(x8*)(base + at + d0) = is_k ? res : raw;
    }
  }
}

// A lane has 8 elements of one token, head and side.
template <class T, int D>
__global__ __launch_bounds__(THREADS) void kv4_read_kernel(Read4Args a) {
  using G = Group4<D>;
  using elem = typename T::elem;
  constexpr int LANES = D / 8;
  const int64_t lanes = (int64_t)a.n_tok * a.kv.kv_heads * 2 * LANES;
  for (int64_t at = (int64_t)blockIdx.x * THREADS + threadIdx.x; at < lanes;
       at += (int64_t)gridDim.x * THREADS) {
    const int sub = (int)(at % LANES);
    const int64_t v = at / LANES;  // token, side, head
    const int kh = (int)(v % a.kv.kv_heads), side = (int)(v / a.kv.kv_heads & 1);
    const int64_t t = v / a.kv.kv_heads >> 1;
    const int slot = a.slots[t], page = slot >> a.kv.page_shift;
    const int off = slot & ((1 << a.kv.page_shift) - 1), tok = off & (GROUP - 1);
    u32x4 x = {0, 0, 0, 0};
    if (slot >= 0 && page < a.kv.n_pages) {
      const char* group = (const char*)a.kv.k + page * a.kv.k_page + kh * a.kv.k_head +
                          (off >> GROUP_SHIFT) * a.kv.k_slot;
      uint32_t code;
      if (side == 0) {
        code = *(const uint32_t*)(group + G::key(tok) + sub * 4);
      } else if constexpr (D == 64) {
        code = *(const uint16_t*)(group + G::value(tok, 2 * sub)) |
               (uint32_t)*(const uint16_t*)(group + G::value(tok, 2 * sub + 1)) << 16;
      } else {
        constexpr int PER = D / 128;
        code = *(const uint32_t*)(group + G::value(tok, sub / PER) + sub % PER * 4);
      }
      const int byte = *(const uint8_t*)(group + (side == 0 ? G::key_scale(tok, sub >> 2)
                                                            : G::value_scale(tok, sub >> 2)));
      x = values8<T>(code, scale_of(byte));
      if (byte == 255) {  // NaN
        const uint32_t nan = pack2<T>(__builtin_nanf(""), __builtin_nanf(""));
        x = (u32x4){nan, nan, nan, nan};
      }
    }
    elem* out = (elem*)(side == 0 ? a.k_out : a.v_out);
    *(u32x4*)(out + t * a.token + kh * a.head + sub * 8) = x;
  }
}

template <class T, int D>
void read(const Read4Args& a, hipStream_t s) {
  const int64_t lanes = (int64_t)a.n_tok * a.kv.kv_heads * 2 * (D / 8);
  const int64_t blocks = (lanes + THREADS - 1) / THREADS, most = 1 << 22;  // 2^30 threads
  kv4_read_kernel<T, D><<<dim3((unsigned)(blocks < most ? blocks : most)), THREADS, 0, s>>>(a);
}

template <class T, int D, bool FP4>
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
  if (a.interleaved) qk_rope_kernel<T, D, true, FP4><<<grid, block, 0, s>>>(a, chunks, per);
  else qk_rope_kernel<T, D, false, FP4><<<grid, block, 0, s>>>(a, chunks, per);
  return hipGetLastError();
}

template <class T, bool FP4>
hipError_t launch_dim(const RopeArgs& a, int head_dim, int n_cu, hipStream_t s) {
  switch (head_dim) {
    case 64: return launch<T, 64, FP4>(a, n_cu, s);
    case 128: return launch<T, 128, FP4>(a, n_cu, s);
    default: return launch<T, 256, FP4>(a, n_cu, s);
  }
}

template <class T>
void read_dim(const Read4Args& a, int head_dim, hipStream_t s) {
  switch (head_dim) {
    case 64: return read<T, 64>(a, s);
    case 128: return read<T, 128>(a, s);
    default: return read<T, 256>(a, s);
  }
}

}  // namespace

hipError_t launch_qk_rope(const RopeArgs& a, int dtype, int head_dim, int n_cu, hipStream_t s) {
  return dtype == FSCHED_BF16 ? launch_dim<Bf16, false>(a, head_dim, n_cu, s)
                              : launch_dim<F16, false>(a, head_dim, n_cu, s);
}

hipError_t launch_qk_rope4(const RopeArgs& a, int dtype, int head_dim, int n_cu, hipStream_t s) {
  return dtype == FSCHED_BF16 ? launch_dim<Bf16, true>(a, head_dim, n_cu, s)
                              : launch_dim<F16, true>(a, head_dim, n_cu, s);
}

hipError_t launch_kv4_read(const Read4Args& a, int dtype, int head_dim, hipStream_t s) {
  if (dtype == FSCHED_BF16) read_dim<Bf16>(a, head_dim, s);
  else read_dim<F16>(a, head_dim, s);
  return hipGetLastError();
}

}  // namespace fs
