// Attention for requests with few rows over a cache of 4 bits: the products, pieces and
// joining of attend_rows.hpp, where a lane's codes become its operands in registers.
//   S^T = K Q^T  a lane takes D/4 neighbouring elements of one key (16 bytes of codes for
//     a D of 128) and one scale or two; the contraction's order is its own, the queries
//     follow it.
//   O^T = V^T P^T  a lane takes a piece (D/16 elements) of the four keys 4h..4h+3 of each
//     of two groups; a conversion gives two neighbouring elements of one key, a byte
//     permute pairs equal elements of two.
// Conversions are exact: an element of 4 bits times its scale is an element of 16.
//
// A unit's loads are little more than a quarter of the 16-bit cache's, so the next unit's are
// under way while one is worked on.  Measured (heads of 128): 512 requests holding 0.73 M
// tokens, 90 us or 4.5 TB/s (the loads alone 82); two of 0.19 M, 44 us or 4.8 TB/s.
#pragma once
#include <hip/hip_runtime.h>

#include "attend_rows.hpp"
#include "fp4.hpp"

namespace fs {

// What a lane loads of a unit: two groups of 16 keys.
template <int D>
struct Unit4 {
  static constexpr int WORDS = D / 32;  // dwords of codes, keys and values alike
  uint32_t k[2][WORDS], v[2][WORDS];
  uint32_t k_scale[2];  // of the lane's one or two blocks
  uint32_t v_scale[2];  // of its four tokens
  uint32_t found;       // keys of the unit that some row sees and the cache holds
};

template <class T, int D, int RT>
__device__ __forceinline__ void attend_rows4(const AttnArgs& a, const RowsPlan& plan, int block,
                                             char* lds) {
  constexpr int KC = D / 32;   // products of a key: 8 elements of each lane
  constexpr int DL = D / 16;   // elements of a value per lane
  using elem = typename T::elem;
  using x8 = typename T::x8;
  using G = Group4<D>;
  using Unit = Unit4<D>;
  const int lane = threadIdx.x & 63;
  const int col = lane & 15, h = lane >> 4;
  const int shift = a.kv.page_shift, page_mask = (1 << shift) - 1;
  // a lane's places in a group
  const uint32_t k_lane = G::key(col) + h * (D / 8), v_lane = G::value(4 * h, col);
  const uint32_t ks_lane = G::key_scale(col, h * (D / 4) / 32);
  const uint32_t vs_lane = G::value_scale(4 * h, col * DL / 32);

  RowsLine line = rows_line(a, plan, 16 * RT, block, lds);
  if (line.me >= line.waves) return;
  if (plan.whole) {  // the tiles that begin in this wave's piece
    line.begin = rows_tile_from(a, line, line.begin);
    line.end = rows_tile_from(a, line, line.end);
  }
  for (int64_t w = line.begin; w < line.end;) {
    const RowsPart part = rows_part(a, line, w);
    // the same in all lanes, and places from them too: scalars
    const int kh = uni_int(part.kh), u0 = uni_int(part.u0), u1 = uni_int(part.u1);
    const int r = uni_int(part.r);
    const Request x = uniform_request(request_of(a, r));
    const Span sp = rows_span(a, x);
    const int rows = rows_of(a, x);
    const int first_own = x.kv - x.q_len;           // own index of the first token
    const int last_own = first_own + min(x.q_len, a.max_q) - 1;
    const int n_keys = min(x.kv, last_own + 1);     // keys past it are seen by none
    const int sink_keys = a.window > 0 ? a.n_sink - a.prefix_len : 0;  // own sinks

    x8 q[RT][KC];
    int top[RT], low[RT];  // a row sees keys low < s <= top, and sinks up to top
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      const int row = t * 16 + col;
      const bool on = row < rows;
      const int i = on ? row / a.group : 0;
      const int qh = kh * a.group + (on ? row - i * a.group : 0);
      const elem* src = (const elem*)a.q + (int64_t)(x.q0 + i) * a.q_token +
                        (int64_t)qh * a.q_head + h * (D / 4);
#pragma unroll
      for (int c = 0; c < KC; ++c) q[t][c] = *(const x8*)(src + c * 8);
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
    const char* base = (const char*)a.kv.k + kh * a.kv.k_head;
    // Keys j .. j + 15 that some row sees, as bits; the page of a group without any is not
    // looked up.
    auto seen = [&](int j) {
      const int n = min(16, n_keys - j);
      uint32_t bits = n > 0 ? (1u << n) - 1 : 0;
      if (a.window > 0) {
        const int from = first_own - a.window + 1 - j;  // the window's first
        const int sinks = min(max(0, sink_keys - j), 16);
        const uint32_t in = from <= 0 ? 0xffff : from > 15 ? 0 : 0xffff & ~((1u << from) - 1);
        bits &= in | ((1u << sinks) - 1);
      }
      return bits;
    };
    auto page_of = [&](int u, int b) {
      const int j = sp.block(u) * UNIT + b * GROUP;
      return seen(j) ? table[j >> shift] : -1;
    };
    // Loads come back in their order: the next unit's pages (then()) are asked for before this
    // one's codes, so that they are not waited for with them (the two batches above, calls:
    // 102.9 -> 100.8, 54.0 -> 52.2 us).
    auto load = [&](int u, const int (&pages)[2], auto then) {
      Unit y;
      y.found = 0;
      const int s0 = sp.block(u) * UNIT;
      const char* group[2];
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const int at = uni_int(pages[b]);
        const bool held = (uint32_t)at < (uint32_t)a.kv.n_pages;
        y.found |= held ? seen(s0 + b * GROUP) << (b * 16) : 0;
        // a group that is not there reads page 0, which exists if any group does
        const uint32_t page = held ? at : 0;
        const uint32_t slot = (uint32_t)(s0 + b * GROUP) & page_mask;
        group[b] = base + page * (uint64_t)a.kv.k_page +
                   (slot >> GROUP_SHIFT) * (uint64_t)a.kv.k_slot;
      }
      then();
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const char* g = group[b];
#pragma unroll
        for (int i = 0; i < Unit::WORDS; ++i) {
          y.k[b][i] = __builtin_nontemporal_load((const uint32_t*)(g + k_lane) + i);
          y.v[b][i] = __builtin_nontemporal_load((const uint32_t*)(g + v_lane) + i);
        }
        y.k_scale[b] = D == 256 ? *(const uint16_t*)(g + ks_lane) : *(const uint8_t*)(g + ks_lane);
        y.v_scale[b] = *(const uint32_t*)(g + vs_lane);
      }
      return y;
    };

    auto work = [&](int u, const Unit& y) {
      const int s0 = sp.block(u) * UNIT;
      const uint32_t found = y.found;
      if (found == 0) return;
      // all 32 keys held, and seen by every row
      const bool full = found == ~0u && s0 + UNIT - 1 <= first_own &&
                        (a.window == 0 || s0 > last_own - a.window || s0 + UNIT <= sink_keys);

      x8 k[2][KC];
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int c = 0; c < KC; ++c) {
          const uint32_t byte = D == 256 ? (y.k_scale[b] >> (c / 4 * 8)) & 255 : y.k_scale[b];
          k[b][c] = __builtin_bit_cast(x8, values8<T>(y.k[b][c], scale_of(byte)));
        }
      const uint32_t mine = found >> (4 * h);  // bits of the lane's keys
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
              const bool see = (bool)((mine >> (b * 16 + i)) & 1) & (key <= top[t]) &
                               ((key > low[t]) | (key < sink_keys));
              s[b][i] = see ? s[b][i] : NEG_INF;
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
        const float at = mu[t] == NEG_INF ? 0.0f : mu[t];
        float e[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          e[j] = exp2_fast(fmaf(s[j >> 2][j & 3], a.scale_log2, -at));
          l[t] += e[j];
          p[t][j] = (elem)e[j];  // the second product's operand (attend_common.hpp)
        }
      }

      uint32_t v_scale[2] = {y.v_scale[0], y.v_scale[1]};
      if (found != ~0u) {
        // where no key is the scale may be NaN, and 0 * NaN is NaN
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (!((mine >> (b * 16 + i)) & 1))
              v_scale[b] = (v_scale[b] & ~(255u << (8 * i))) | 127u << (8 * i);
      }
      float vs[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) vs[j] = scale_of((v_scale[j >> 2] >> (8 * (j & 3))) & 255);
      auto values = [&](auto at) {  // elements 2i and 2i + 1 of the lane's 8 keys
        constexpr int i = decltype(at)::value;
        uint32_t z[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const uint32_t* v = y.v[j >> 2];
          if constexpr (D == 64)
            z[j] = j & 1 ? values2<T, 2 + (i & 1)>(v[(j & 3) >> 1], vs[j])
                         : values2<T, i & 1>(v[(j & 3) >> 1], vs[j]);
          else
            z[j] = values2<T, i & 3>(v[(j & 3) * (D / 128) + (i >> 2)], vs[j]);
        }
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          u32x4 f;
#pragma unroll
          for (int n = 0; n < 4; ++n)
            f[n] = __builtin_amdgcn_perm(z[2 * n + 1], z[2 * n],
                                         e ? 0x07060302u : 0x05040100u);
          const x8 vt = __builtin_bit_cast(x8, f);
#pragma unroll
          for (int t = 0; t < RT; ++t) o[t][2 * i + e] = T::mfma16(vt, p[t], o[t][2 * i + e]);
        }
      };
      each<DL / 2>(values);
    };

    // units u0 .. last, two in turn: while one is worked on the next one's loads are under
    // way, and its own place is loaded again behind it.  Pages are looked up before that.
    const int last = sp.blocks > 0 && a.kv.n_pages > 0 ? u1 : u0;
    Unit ready[2];
    int pages[2] = {-1, -1};
    auto look_up = [&](int u) {
      if (u < last) {
#pragma unroll
        for (int b = 0; b < 2; ++b) pages[b] = page_of(u, b);
      }
    };
    look_up(u0);
    if (u0 < last) ready[0] = load(u0, pages, [&] { look_up(u0 + 1); });
    if (u0 + 1 < last) ready[1] = load(u0 + 1, pages, [&] { look_up(u0 + 2); });
    for (int u = u0; u < last; u += 2) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        if (u + i >= last) break;
        work(u + i, ready[i]);
        if (u + i + 2 < last) ready[i] = load(u + i + 2, pages, [&] { look_up(u + i + 3); });
      }
    }
    rows_write<T, D, RT>(a, plan, line, part, w, x, rows, o, mu, l);
    w += u1 - u0;
  }
}

}  // namespace fs
