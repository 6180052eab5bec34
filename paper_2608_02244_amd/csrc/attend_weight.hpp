// Attention weight of held tokens (fsched_attend_weight, fsched_attend4_weight):
//   weight[r][j] += sum over the new tokens i of request r and the query heads h that see
//   key j of exp(scale q_ih . k_j - lse_ih)
//
// Q K^T with rows of Q as the first operand: 16 rows x 16 keys, a lane holds 4 rows of one
// key, so that a key's sum needs two exchanges at the end and no more.  The keys of all
// requests form one line of units of 64; a block takes an equal piece of it, up to 256 keys
// of one request at once, whose units and key heads its waves share out; their sums meet in
// LDS.  A key is one block's, so nothing is added twice or in an order that varies.
#pragma once
#include <hip/hip_runtime.h>

#include "attend_common.hpp"
#include "fp4.hpp"

namespace fs {

constexpr int WEIGHT_UNIT = 64, WEIGHT_UNITS = 4, WEIGHT_KEYS = WEIGHT_UNIT * WEIGHT_UNITS;
constexpr float LOG2E = 1.4426950408889634f;

// What a lane loads of one key: its share of the elements, D/4.
template <int D, bool FP4>
struct WeightKey {
  static constexpr int WORDS = FP4 ? D / 32 : D / 8;
  uint32_t w[WORDS];
  uint32_t scale;
};

template <class T, int D, bool FP4>
__global__ __launch_bounds__(ATT_THREADS, 2) void weight_rows_kernel(WeightArgs wa) {
  constexpr int KC = D / 32;
  using elem = typename T::elem;
  using x8 = typename T::x8;
  using Key = WeightKey<D, FP4>;
  using G = Group4<D>;
  const AttnArgs& a = wa.at;
  __shared__ float sums[ATT_WAVES][WEIGHT_KEYS];
  extern __shared__ __attribute__((aligned(16))) char lds[];
  int64_t* wave_sum = (int64_t*)lds;       // [ATT_WAVES]
  int64_t* before = wave_sum + ATT_WAVES;  // [n_req + 1] units before request r
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, col = lane & 15, h = lane >> 4;
  const int shift = a.kv.page_shift, page_mask = (1 << shift) - 1;

  auto span = [&](const Request& x) {
    const int p0 = x.kv - x.q_len, n = min(x.q_len, a.max_q);
    Span s = span_of<WEIGHT_UNIT>(p0, p0 + n - 1, x.kv, a.window, a.n_sink, a.prefix_len);
    if (n <= 0) s.blocks = 0;
    return s;
  };
  {
    const int n = a.n_req, per = (n + ATT_THREADS - 1) / ATT_THREADS;
    const int r0 = min(n, tid * per), r1 = min(n, r0 + per);
    int64_t sum = 0;
    for (int r = r0; r < r1; ++r) {
      const int u = span(request_of(a, r)).blocks;
      before[r] = u;
      sum += u;
    }
    int64_t x = sum;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int64_t y = __shfl_up(x, d);
      if (lane >= d) x += y;
    }
    if (lane == 63) wave_sum[wave] = x;
    __syncthreads();
    for (int w = 0; w < wave; ++w) x += wave_sum[w];
    int64_t at = x - sum;
    for (int r = r0; r < r1; ++r) {
      const int64_t u = before[r];
      before[r] = at;
      at += u;
    }
    if (tid == ATT_THREADS - 1) before[n] = at;
    __syncthreads();
  }
  const int64_t total = before[a.n_req];
  const int64_t begin = total * blockIdx.x / gridDim.x, end = total * (blockIdx.x + 1) / gridDim.x;

  for (int64_t w = begin; w < end;) {
    int lo = 0, hi = a.n_req;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (before[mid] <= w) lo = mid;
      else hi = mid;
    }
    const int r = uni_int(lo);
    const Request x = request_of(a, r);
    const Span sp = span(x);
    const int u0 = (int)(w - before[r]);
    const int units = (int)min((int64_t)WEIGHT_UNITS, min(end, before[r + 1]) - w);
    const int first_own = x.kv - x.q_len, n_new = min(x.q_len, a.max_q);
    const int last_own = first_own + n_new - 1;
    const int n_keys = min(x.kv, last_own + 1);
    const int sink_keys = a.window > 0 ? a.n_sink - a.prefix_len : 0;
    const int rows = n_new * a.group;
    const int32_t* table = a.table + (int64_t)r * a.width;

#pragma unroll
    for (int i = 0; i < WEIGHT_UNITS; ++i) sums[wave][i * 64 + lane] = 0.0f;

    // items: half a unit (32 keys) of one key head, heads first
    const int halves = 2 * units, items = halves * a.kv.kv_heads;
    const int i0 = items * wave / ATT_WAVES, i1 = items * (wave + 1) / ATT_WAVES;
    for (int i = i0; i < i1;) {
      const int kh = i / halves, j0 = i - kh * halves, j1 = min(halves, j0 + (i1 - i));
      i += j1 - j0;
      const char* kbase = FP4 ? (const char*)a.kv.k + kh * a.kv.k_head
                              : (const char*)((const elem*)a.kv.k + kh * a.kv.k_head);
      auto key_of = [&](int j) { return sp.block(u0 + (j >> 1)) * WEIGHT_UNIT + (j & 1) * 32; };
      for (int row0 = 0; row0 < rows; row0 += 16) {
        // this lane's operand: row row0 + col; its results: rows row0 + 4h + 0..3
        x8 q[KC];
        {
          const int row = min(row0 + col, rows - 1), tok = row / a.group;
          const elem* src = (const elem*)a.q + (int64_t)(x.q0 + tok) * a.q_token +
                            (int64_t)(kh * a.group + row - tok * a.group) * a.q_head;
#pragma unroll
          for (int c = 0; c < KC; ++c)
            q[c] = *(const x8*)(src + (FP4 ? h * (D / 4) + c * 8
                                           : h * 16 + (c >> 1) * 64 + (c & 1) * 8));
        }
        float lse[4];
        int top[4], low[4];
        const int tok0 = row0 / a.group, tok1 = min(row0 + 15, rows - 1) / a.group;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int row = row0 + 4 * h + e;
          const bool on = row < rows;
          const int tok = (on ? row : 0) / a.group;
          const float v = on ? wa.lse[(int64_t)(x.q0 + tok) * a.q_heads + kh * a.group + row -
                                      tok * a.group]
                             : NEG_INF;
          // a row that sees nothing gives nothing
          lse[e] = v == NEG_INF ? -NEG_INF : v * LOG2E;
          top[e] = on ? first_own + tok : -1;
          low[e] = a.window > 0 ? top[e] - a.window : -0x7fffffff - 1;
        }
        for (int j = j0; j < j1; ++j) {
          const int s0 = key_of(j);
          if (s0 > first_own + tok1) continue;  // seen by none of these rows
          if (a.window > 0 && s0 + 31 <= first_own + tok0 - a.window && s0 >= sink_keys) continue;
          const bool full = s0 + 31 <= first_own + tok0 && (a.window == 0 ||
                            s0 > first_own + tok1 - a.window || s0 + 32 <= sink_keys);
#pragma unroll
          for (int b = 0; b < 2; ++b) {
            const int key = s0 + b * 16 + col;
            const bool in = key < n_keys && (a.window == 0 || key > first_own - a.window ||
                                             key < sink_keys);
            const int page = in ? table[key >> shift] : -1;
            const bool held = (uint32_t)page < (uint32_t)a.kv.n_pages;
            x8 k[KC];
            if (held) {
              const int slot = key & page_mask;
              if constexpr (FP4) {
                const char* g = kbase + page * (uint64_t)a.kv.k_page +
                                (slot >> GROUP_SHIFT) * (uint64_t)a.kv.k_slot;
                const int t = slot & (GROUP - 1);
                const uint32_t* codes = (const uint32_t*)(g + G::key(t) + h * (D / 8));
                const char* sc = g + G::key_scale(t, h * (D / 4) / 32);
                const uint32_t bytes = D == 256 ? *(const uint16_t*)sc : *(const uint8_t*)sc;
#pragma unroll
                for (int c = 0; c < KC; ++c)
                  k[c] = __builtin_bit_cast(
                      x8, values8<T>(codes[c], scale_of((bytes >> (c / 4 * 8)) & 255)));
              } else {
                const elem* src = (const elem*)kbase + page * a.kv.k_page + slot * a.kv.k_slot +
                                  h * 16;
#pragma unroll
                for (int c = 0; c < KC; ++c)
                  k[c] = *(const x8*)(src + (c >> 1) * 64 + (c & 1) * 8);
              }
            } else {
#pragma unroll
              for (int c = 0; c < KC; ++c) k[c] = x8{};
            }
            f32x4 s = {0, 0, 0, 0};
#pragma unroll
            for (int c = 0; c < KC; ++c) s = T::mfma16(q[c], k[c], s);
            float sum = 0.0f;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const bool see = full || (key <= top[e] && (key > low[e] || key < sink_keys));
              const float p = exp2_fast(fmaf(s[e], a.scale_log2, -lse[e]));
              sum += see ? p : 0.0f;
            }
            sum = sum_xor32(sum_xor16(held ? sum : 0.0f));
            if (h == 0) sums[wave][(j >> 1) * 64 + (j & 1) * 32 + b * 16 + col] += sum;
          }
        }
      }
    }
    __syncthreads();
    if (tid < units * WEIGHT_UNIT) {
      const int key = sp.block(u0 + tid / WEIGHT_UNIT) * WEIGHT_UNIT + tid % WEIGHT_UNIT;
      if (key < n_keys) {
        float* at = wa.weight + (int64_t)r * wa.weight_stride + key;
        *at += (sums[0][tid] + sums[1][tid]) + (sums[2][tid] + sums[3][tid]);
      }
    }
    __syncthreads();
    w += units;
  }
}

}  // namespace fs
