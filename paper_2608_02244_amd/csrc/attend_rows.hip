// Attention for requests with few rows: decode steps and drafts.
//
// One tile is a request and a key head; its rows are the tokens times the query
// heads that read this key head, up to 16 (or 32).  Every key and value is read
// once for all of them, straight from the cache into the registers that feed the
// matrix unit, so the kernel is bound by the bytes of the cache:
//   S^T = K Q^T  16 keys x 16 rows; a lane's 16 bytes of a key are its operand.
//   O^T = V^T P^T  the contraction runs over 32 keys in an order of its own choice
//     (lane group h: keys 4h..4h+3 and 16+4h..16+4h+3), which is the one in which
//     the scores leave the first product, so P stays in its lanes; the values of
//     a lane's 8 keys, D/16 neighbouring elements each, become operands by packing
//     equal elements of two keys (one byte permute each).
// A row is a lane's column throughout: scaling it needs no exchange.
//
// The keys of all tiles form one line of units of 128 keys, cut into equal pieces,
// one per block (4 waves, 32 keys of a unit each): however uneven the lengths, all
// blocks end together, and one long request spreads over the device.  Pieces that
// cover a whole tile write its result; the others write parts, which a second
// launch joins.
#include <hip/hip_runtime.h>

#include "attend_common.hpp"
#include "attend_rows.hpp"

namespace fs {
namespace {

constexpr int THREADS = 256, WAVES = 4;
constexpr int WAVE_KEYS = 32, UNIT = WAVES * WAVE_KEYS;

// Blocks per compute unit that the registers allow (head_dim, row tiles).
constexpr int occupancy(int D, int RT) { return D == 256 || (D == 128 && RT == 2) ? 2 : 3; }

template <int D, int RT>
struct Merge {  // LDS of a block's four partial results
  float o[WAVES][16 * RT][D + 4];
  float2 ml[WAVES][16 * RT];
};

template <class T, int D, int RT>
__global__ __launch_bounds__(THREADS, occupancy(D, RT)) void attend_rows_kernel(AttnArgs a,
                                                                                RowsPlan plan) {
  constexpr int KC = D / 32;   // 32-element chunks of a key
  constexpr int DL = D / 16;   // elements of a value per lane
  constexpr int VW = DL / 2;   // dwords of them
  using elem = typename T::elem;
  using x8 = typename T::x8;
  extern __shared__ __attribute__((aligned(16))) char lds[];
  Merge<D, RT>& merge = *(Merge<D, RT>*)lds;
  int64_t* before = (int64_t*)(lds + sizeof(Merge<D, RT>));  // [n_req + 1] units before request r
  __shared__ int64_t wave_sum[WAVES];

  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int col = lane & 15, h = lane >> 4;
  const int shift = a.kv.page_shift, page_mask = (1 << shift) - 1;

  auto rows_of = [&](const Request& x) { return min(x.q_len, a.max_q) * a.group; };
  auto mine = [&](const Request& x) { return x.q_len > 0 && rows_of(x) <= 16 * RT; };
  auto span = [&](const Request& x) {
    const int p0 = x.kv - x.q_len;  // own index of the first token
    return span_of<UNIT>(p0, p0 + min(x.q_len, a.max_q) - 1, x.kv, a.window, a.n_sink,
                         a.prefix_len);
  };

  // units before each request: a tile without a visible key is one unit all the same
  {
    const int n = a.n_req, per = (n + THREADS - 1) / THREADS;
    const int r0 = min(n, tid * per), r1 = min(n, r0 + per);
    int64_t sum = 0;
    for (int r = r0; r < r1; ++r) {
      const Request x = request_of(a, r);
      const int u = mine(x) ? max(1, span(x).blocks) : 0;
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
    if (tid == THREADS - 1) before[n] = at;
    __syncthreads();
  }
  const int64_t per_head = before[a.n_req];
  const int64_t total = per_head * a.kv.kv_heads;
  const int64_t piece = (total + plan.blocks - 1) / plan.blocks;
  const int64_t begin = (int64_t)blockIdx.x * piece;
  const int64_t end = min(total, begin + piece);

  for (int64_t w = begin; w < end;) {
    const int kh = (int)(w / per_head);
    const int64_t rest = w - kh * per_head;
    int lo = 0, hi = a.n_req;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (before[mid] <= rest) lo = mid;
      else hi = mid;
    }
    const int r = lo;
    const int units = (int)(before[r + 1] - before[r]);
    const int u0 = (int)(rest - before[r]);
    const int u1 = (int)min((int64_t)units, u0 + (end - w));
    const Request x = request_of(a, r);
    const Span sp = span(x);
    const int rows = rows_of(x);
    const int first_own = x.kv - x.q_len;           // own index of the first token
    const int last_own = first_own + min(x.q_len, a.max_q) - 1;
    const int n_keys = min(x.kv, last_own + 1);     // keys past it are seen by none
    const int sink_keys = a.window > 0 ? a.n_sink - a.prefix_len : 0;  // own sinks

    // rows of this lane, and their queries
    x8 q[RT][KC];
    int top[RT], low[RT];  // a row sees keys low < s <= top, and sinks up to top
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      const int row = t * 16 + col;
      const bool on = row < rows;
      const int i = on ? row / a.group : 0;
      const int qh = kh * a.group + (on ? row - i * a.group : 0);
      const elem* src = (const elem*)a.q + (int64_t)(x.q0 + i) * a.q_token +
                        (int64_t)qh * a.q_head + h * 8;
#pragma unroll
      for (int c = 0; c < KC; ++c) q[t][c] = *(const x8*)(src + c * 32);
      top[t] = on ? first_own + i : -1;
      low[t] = a.window > 0 ? top[t] - a.window : -0x7fffffff - 1;
    }

    f32x4 o[RT][DL];
    float mu[RT], l[RT];
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      mu[t] = NEG_INF;
      l[t] = 0.0f;
#pragma unroll
      for (int d = 0; d < DL; ++d) o[t][d] = (f32x4){0, 0, 0, 0};
    }

    const int32_t* table = a.table + (int64_t)r * a.width;
    const elem* kbase = (const elem*)a.kv.k + kh * a.kv.k_head + h * 8;
    const elem* vbase = (const elem*)a.kv.v + kh * a.kv.v_head + col * DL;
    // page of key s0 + (lane mod 32), -1 where no row sees a key
    auto page_at = [&](int u) {
      const int s = sp.block(u) * UNIT + wave * WAVE_KEYS + (lane & 31);
      int p = -1;
      if (u < u1 && s < n_keys &&
          (a.window == 0 || s > first_own - a.window || s < sink_keys))
        p = table[s >> shift];
      return (uint32_t)p < (uint32_t)a.kv.n_pages ? p : -1;
    };

    int page = sp.blocks > 0 ? page_at(u0) : -1;
    for (int u = u0; u < u1; ++u) {
      const int s0 = sp.block(u) * UNIT + wave * WAVE_KEYS;
      const int here = page;
      page = page_at(u + 1);
      const uint64_t found = __ballot(here >= 0);
      if (found == 0) continue;
      // all 32 keys held, and seen by every row
      const bool full = found == ~0ull && s0 + WAVE_KEYS - 1 <= first_own &&
                        (a.window == 0 || s0 > last_own - a.window ||
                         s0 + WAVE_KEYS <= sink_keys);

      x8 k[2][KC];
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const int pg = max(0, __shfl(here, b * 16 + col));
        const elem* src = kbase + pg * a.kv.k_page +
                          ((s0 + b * 16 + col) & page_mask) * a.kv.k_slot;
#pragma unroll
        for (int c = 0; c < KC; ++c) k[b][c] = *(const x8*)(src + c * 32);
      }
      uint32_t v[8][VW];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int key = (j & 3) + 4 * h + (j >> 2) * 16;
        const int pg = __shfl(here, key);
        const elem* src = vbase + max(0, pg) * a.kv.v_page +
                          ((s0 + key) & page_mask) * a.kv.v_slot;
        if constexpr (VW == 2) {
          const u32x2 y = *(const u32x2*)src;
          v[j][0] = y[0];
          v[j][1] = y[1];
        } else {
#pragma unroll
          for (int i = 0; i < VW; i += 4) {
            const u32x4 y = *(const u32x4*)(src + 2 * i);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[j][i + e] = y[e];
          }
        }
        if (!full && pg < 0) {  // what sits there may be anything: 0 * NaN would be NaN
#pragma unroll
          for (int i = 0; i < VW; ++i) v[j][i] = 0;
        }
      }

      x8 p[RT];
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        f32x4 s[2];
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          s[b] = (f32x4){0, 0, 0, 0};
#pragma unroll
          for (int c = 0; c < KC; ++c) s[b] = T::mfma16(k[b][c], q[t][c], s[b]);
        }
        if (!full) {
#pragma unroll
          for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int key = s0 + b * 16 + 4 * h + i;
              const bool see = ((found >> (b * 16 + 4 * h + i)) & 1) && key <= top[t] &&
                               (key > low[t] || key < sink_keys);
              if (!see) s[b][i] = NEG_INF;
            }
        }
        float mx = fmaxf(fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3])),
                         fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3])));
        mx = max_xor32(max_xor16(mx)) * a.scale_log2 - BIAS<T>;
        if (__ballot(mx > mu[t] + TAU)) {
          const float to = mx > mu[t] + TAU ? mx : mu[t];
          const float f = part_scale(mu[t], to);
          mu[t] = to;
          l[t] *= f;
#pragma unroll
          for (int d = 0; d < DL; ++d) o[t][d] *= f;
        }
        const float base = mu[t] == NEG_INF ? 0.0f : mu[t];
        float e[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          e[j] = exp2_fast(fmaf(s[j >> 2][j & 3], a.scale_log2, -base));
          l[t] += e[j];
          p[t][j] = (elem)e[j];  // rounded to the type of the values, as the products need
        }
      }

#pragma unroll
      for (int d = 0; d < DL; ++d) {
        const uint32_t pick = d & 1 ? 0x07060302u : 0x05040100u;
        u32x4 y;
#pragma unroll
        for (int i = 0; i < 4; ++i)
          y[i] = __builtin_amdgcn_perm(v[2 * i + 1][d >> 1], v[2 * i][d >> 1], pick);
        const x8 vt = __builtin_bit_cast(x8, y);
#pragma unroll
        for (int t = 0; t < RT; ++t) o[t][d] = T::mfma16(vt, p[t], o[t][d]);
      }
    }

    // join the four waves: each result element is summed by one thread
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      const float sum = sum_xor32(sum_xor16(l[t]));
      if (h == 0) merge.ml[wave][t * 16 + col] = make_float2(mu[t], sum);
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int d = 0; d < DL; d += 4) {
          const f32x4 y = {o[t][d][i], o[t][d + 1][i], o[t][d + 2][i], o[t][d + 3][i]};
          *(f32x4*)&merge.o[wave][t * 16 + col][(4 * h + i) * DL + d] = y;
        }
    }
    __syncthreads();
    const bool whole = u0 == 0 && u1 == units;
    const int slot = 2 * blockIdx.x + (w != begin);
    if (u0 == 0 && tid == 0) {
      RowsTile d;
      d.first = slot;
      d.block = blockIdx.x;
      d.count = (int)((w + units - 1) / piece) - (int)blockIdx.x + 1;
      d.pad = 0;
      plan.tiles[(int64_t)kh * a.n_req + r] = d;
    }
    for (int i = tid; i < rows * (D / 8); i += THREADS) {
      const int row = i / (D / 8), d0 = (i % (D / 8)) * 8;
      float m = NEG_INF, sum = 0.0f, y[8] = {};
#pragma unroll
      for (int v4 = 0; v4 < WAVES; ++v4) m = fmaxf(m, merge.ml[v4][row].x);
#pragma unroll
      for (int v4 = 0; v4 < WAVES; ++v4) {
        const float2 ml = merge.ml[v4][row];
        const float f = part_scale(ml.x, m);
        sum += ml.y * f;
#pragma unroll
        for (int e = 0; e < 8; e += 4) {
          const f32x4 z = *(const f32x4*)&merge.o[v4][row][d0 + e];
#pragma unroll
          for (int g = 0; g < 4; ++g) y[e + g] += z[g] * f;
        }
      }
      if (whole && !plan.keep_parts) {
        const int tok = row / a.group, qh = kh * a.group + row - tok * a.group;
        const float inv = sum > 0.0f ? 1.0f / sum : sum == 0.0f ? 0.0f : sum;
        x8 out;
#pragma unroll
        for (int e = 0; e < 8; ++e) out[e] = (elem)(y[e] * inv);
        *(x8*)((elem*)a.out + (int64_t)(x.q0 + tok) * a.o_token + (int64_t)qh * a.o_head + d0) =
            out;
        if (a.lse && d0 == 0)
          a.lse[(int64_t)(x.q0 + tok) * a.q_heads + qh] = (m + log2f(sum)) * LN2;
      } else {
        const int64_t at = (int64_t)slot * (16 * RT) + row;
        float* dst = plan.part_o + at * D + d0;
        *(f32x4*)dst = (f32x4){y[0], y[1], y[2], y[3]};
        *(f32x4*)(dst + 4) = (f32x4){y[4], y[5], y[6], y[7]};
        if (d0 == 0) plan.part_ml[at] = make_float2(m, sum);
      }
    }
    __syncthreads();
    w += u1 - u0;
  }
}

template <class T, int D, int RT>
hipError_t launch(const AttnArgs& a, const RowsPlan& p, hipStream_t s) {
  const size_t lds = sizeof(Merge<D, RT>) + (size_t)(a.n_req + 1) * sizeof(int64_t);
  if (lds > 64 * 1024) {
    const hipError_t e = hipFuncSetAttribute((const void*)attend_rows_kernel<T, D, RT>,
                                             hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return e;
  }
  attend_rows_kernel<T, D, RT><<<dim3((unsigned)p.blocks), dim3(THREADS), lds, s>>>(a, p);
  return hipGetLastError();
}

template <class T>
hipError_t launch_shape(const AttnArgs& a, const RowsPlan& p, int head_dim, hipStream_t s) {
  switch (head_dim) {
    case 64: return p.row_tiles == 1 ? launch<T, 64, 1>(a, p, s) : launch<T, 64, 2>(a, p, s);
    case 128: return p.row_tiles == 1 ? launch<T, 128, 1>(a, p, s) : launch<T, 128, 2>(a, p, s);
    default: return launch<T, 256, 1>(a, p, s);
  }
}

}  // namespace

int rows_blocks(int head_dim, int row_tiles, int n_cu) {
  return (n_cu > 0 ? n_cu : 256) * occupancy(head_dim, row_tiles);
}

hipError_t launch_attend_rows(const AttnArgs& a, const RowsPlan& p, int dtype, int head_dim,
                              hipStream_t s) {
  return dtype == FSCHED_BF16 ? launch_shape<Bf16>(a, p, head_dim, s)
                              : launch_shape<F16>(a, p, head_dim, s);
}

}  // namespace fs
