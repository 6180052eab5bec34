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
// The keys of all tiles form one line of units of 32 keys, cut into equal pieces, one
// per wave: however uneven the lengths, all waves end together, and one long request
// spreads over the device.  A wave works alone (no barrier, nothing shared after the
// first sums), so while one changes tiles the others of its unit keep loads in flight.
// Pieces that cover a whole tile write its result; the others write parts, which a
// second launch joins.  A wave has two parts at most, the tiles at its piece's ends;
// behind a shared prefix, where whole tiles are parts too and a piece may hold any
// number of them, those have a slot of their own per tile.
//
// Measured (heads of 128, bf16): 512 requests holding 0.73 M tokens, 262 us or 5.7 TB/s;
// 64 requests, 51 us or 5.2 TB/s.  Waves that work alone took 53 us there, blocks of four
// that share a piece behind barriers 69 us.
#pragma once
#include <hip/hip_runtime.h>

#include "attend_common.hpp"

namespace fs {

// A tile's parts: written by the wave that begins the tile.
struct RowsTile {
  int32_t first;  // slot of its first part
  int32_t wave;   // wave that wrote it; the others are slots 2 (wave + 1), 2 (wave + 2), ..
  int32_t count;  // parts; 1: a whole tile (the result itself unless keep_parts)
  int32_t pad;
};

struct RowsPlan {
  int32_t waves;        // of the launch
  int32_t row_tiles;    // 16-row tiles of a request and key head (1 or 2)
  int32_t slot_rows;    // rows of a part's slot
  int32_t most_parts;   // of a tile, on average
  int32_t keep_parts;   // 1: results join with those of the prefix, written as parts
  int32_t whole;        // 1: no tile is cut (a cache of 4 bits; nothing to join then)
  float* part_o;        // [slots][slot_rows][head_dim]; slots: 2 per wave, then with
                        // keep_parts one per tile, for those that lie in one piece
  float2* part_ml;      // [slots][slot_rows] (mu, l)
  RowsTile* tiles;      // [kv_heads][n_req]
};

constexpr int UNIT = 32;       // keys of a unit
// Parts of a tile, on average.  More spread a lone long request over more waves, and cost
// the join more.  One request, heads of 128, a call with 8 / 32 / 128 / 256 parts at most:
//   131,072 tokens, 8 key heads   890 / 245 /  97 / 106 us (5.5 TB/s at 128)
//    16,384 tokens, 8 key heads   120 /  45 /  27 /  36 us
//    65,536 tokens, 1 key head    436 / 119 /  49 /  42 us
//     4,096 tokens, 1 key head     35 /  17 /  18 /  18 us
constexpr int MOST_PARTS = 128;
// Over a cache of 4 bits, whose units take less time, two requests of 95,000 tokens and 8 key
// heads: 57 us with 128, 55 with 256 (that is all waves there).
constexpr int MOST_PARTS4 = 256;

// Blocks per compute unit.  Fewer waves have longer pieces, more of them more loads under
// way.  The registers would allow 4 with heads of 64 and 3 with heads of 128 (one row tile,
// pages of 16 and more); two with heads of 256 would spill to scratch.  Calls in bf16 with
// 1 / 2 / 3 / 4 blocks, us:
//   heads of 128   512 requests, 0.73 M tokens, 4 key heads   262 / 251 / 275
//                  64 requests, 65,000 tokens, 8 key heads     57 /  56 /  58
//   heads of  64   400 requests, 0.57 M tokens, 8 key heads     - / 202 / 205 / 205
//                  64 requests                                  - /  35 /  35 /  36
//   heads of 256   64 requests, pages of 16 and of 8          108 / 117, 107 / 126
//                  64 drafts; one request of 131,072 tokens   122 / 136, 218 / 211
// Over a cache of 4 bits, whose loads are shorter, as many as the registers leave (a second
// row tile takes one place of heads of 64 and 128).
constexpr int rows_occupancy(int D, bool fp4, int row_tiles) {
  if (fp4) return D == 256 ? 2 : (D == 64 ? 4 : 3) - (row_tiles == 2);
  return D == 64 ? 3 : D == 128 ? 2 : 1;
}

// The line of units and a wave's piece of it.
struct RowsLine {
  const int64_t* before;  // [n_req + 1] units before request r, of one key head (LDS)
  int64_t per_head, total, waves;
  int me;                 // this wave; at or past `waves`: without work
  int64_t begin, end;     // its units

  static __device__ __forceinline__ int64_t quotient(int64_t x, int64_t y) {
    // a 64-bit division is some 130 instructions
    return ((x | y) >> 32) == 0 ? (int64_t)((uint32_t)x / (uint32_t)y) : x / y;
  }
  __device__ __forceinline__ int wave_of(int64_t unit) const {
    return (int)quotient((unit + 1) * waves - 1, total);
  }
};

__device__ __forceinline__ int rows_of(const AttnArgs& a, const Request& x) {
  return min(x.q_len, a.max_q) * a.group;
}

__device__ __forceinline__ Span rows_span(const AttnArgs& a, const Request& x) {
  const int p0 = x.kv - x.q_len;  // own index of the first token
  return span_of<UNIT>(p0, p0 + min(x.q_len, a.max_q) - 1, x.kv, a.window, a.n_sink,
                       a.prefix_len);
}

// Units before each request (a tile without a visible key is one unit all the same), and
// the piece of this wave.  All threads of the block call it.
__device__ __forceinline__ RowsLine rows_line(const AttnArgs& a, const RowsPlan& plan, int most,
                                              int block, char* lds) {
  int64_t* wave_sum = (int64_t*)lds;  // [ATT_WAVES]
  int64_t* before = wave_sum + ATT_WAVES;  // [n_req + 1] units before request r
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  auto mine = [&](const Request& x) { return x.q_len > 0 && rows_of(a, x) <= most; };
  {
    const int n = a.n_req, per = (n + ATT_THREADS - 1) / ATT_THREADS;
    const int r0 = min(n, tid * per), r1 = min(n, r0 + per);
    int64_t sum = 0;
    for (int r = r0; r < r1; ++r) {
      const Request x = request_of(a, r);
      const int u = mine(x) ? max(1, rows_span(a, x).blocks) : 0;
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
  RowsLine l;
  l.before = before;
  l.per_head = before[a.n_req];
  l.total = l.per_head * a.kv.kv_heads;
  // Waves with work: a few tiles are not cut finer than their parts are worth reading
  // again.  Wave i takes units i total / waves .. (i + 1) total / waves.
  l.waves = min(min((int64_t)plan.waves, l.total),
                (int64_t)plan.most_parts * a.n_req * a.kv.kv_heads);
  l.me = uni_int(block * ATT_WAVES + wave);
  l.begin = l.end = 0;
  if (l.me < l.waves) {
    l.begin = RowsLine::quotient(l.me * l.total, l.waves);
    l.end = RowsLine::quotient((l.me + 1) * l.total, l.waves);
  }
  return l;
}

// The tile of a unit, and what of it lies in the wave's piece.
struct RowsPart {
  int kh, r, units, u0, u1;  // units u0 .. u1 of the tile's `units`
};

__device__ __forceinline__ RowsPart rows_part(const AttnArgs& a, const RowsLine& l, int64_t w) {
  RowsPart p;
  p.kh = (int)RowsLine::quotient(w, l.per_head);
  const int64_t rest = w - p.kh * l.per_head;
  int lo = 0, hi = a.n_req;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (l.before[mid] <= rest) lo = mid;
    else hi = mid;
  }
  p.r = lo;
  p.units = (int)(l.before[lo + 1] - l.before[lo]);
  p.u0 = (int)(rest - l.before[lo]);
  p.u1 = (int)min((int64_t)p.units, p.u0 + (l.end - w));
  return p;
}

// The first unit from w on that begins a tile.
__device__ __forceinline__ int64_t rows_tile_from(const AttnArgs& a, const RowsLine& l,
                                                  int64_t w) {
  if (w >= l.total) return l.total;
  const RowsPart p = rows_part(a, l, w);
  return p.u0 == 0 ? w : w - p.u0 + p.units;
}

// A part's end: the result of a tile that lies whole in the wave's piece, else a part for
// the join.  A lane holds 4 DL neighbouring elements of its rows, from 4 DL h on.
template <class T, int D, int RT>
__device__ __forceinline__ void rows_write(const AttnArgs& a, const RowsPlan& plan,
                                           const RowsLine& line, const RowsPart& at_unit,
                                           int64_t w, const Request& x, int rows,
                                           const f32x4 (&o)[RT][D / 16], const float (&mu)[RT],
                                           const float (&l)[RT]) {
  constexpr int DL = D / 16;
  using elem = typename T::elem;
  const int lane = threadIdx.x & 63, col = lane & 15, h = lane >> 4, kh = at_unit.kh;
  const bool whole = at_unit.u0 == 0 && at_unit.u1 == at_unit.units;
  const int64_t tile = (int64_t)kh * a.n_req + at_unit.r;
  const int64_t slot = whole && plan.keep_parts ? 2 * (int64_t)plan.waves + tile
                                                : 2 * (int64_t)line.me + (w != line.begin);
  if (at_unit.u0 == 0 && lane == 0) {
    RowsTile d;
    d.first = (int32_t)slot;
    d.wave = line.me;
    d.count = line.wave_of(w + at_unit.units - 1) - line.me + 1;
    d.pad = 0;
    plan.tiles[tile] = d;
  }
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    const int row = t * 16 + col;
    const float sum = sum_xor32(sum_xor16(l[t]));
    if (row >= rows) continue;
    if (whole && !plan.keep_parts) {
      const int tok = row / a.group, qh = kh * a.group + row - tok * a.group;
      const float inv = sum > 0.0f ? 1.0f / sum : sum == 0.0f ? 0.0f : sum;
      uint32_t y[2 * DL];
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int d = 0; d < DL; d += 2)
          y[(i * DL + d) / 2] = pack2<T>(o[t][d][i] * inv, o[t][d + 1][i] * inv);
      elem* dst = (elem*)a.out + (int64_t)(x.q0 + tok) * a.o_token + (int64_t)qh * a.o_head +
                  4 * DL * h;
#pragma unroll
      for (int i = 0; i < 2 * DL; i += 4)
        *(u32x4*)(dst + 2 * i) = (u32x4){y[i], y[i + 1], y[i + 2], y[i + 3]};
      if (a.lse && h == 0)
        a.lse[(int64_t)(x.q0 + tok) * a.q_heads + qh] = (mu[t] + log2f(sum)) * LN2;
    } else {
      const int64_t at = slot * plan.slot_rows + row;
      float* dst = plan.part_o + at * D + 4 * DL * h;
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int d = 0; d < DL; d += 4)
          *(f32x4*)(dst + i * DL + d) =
              (f32x4){o[t][d][i], o[t][d + 1][i], o[t][d + 2][i], o[t][d + 3][i]};
      if (h == 0) plan.part_ml[at] = make_float2(mu[t], sum);
    }
  }
}

// WIDE: pages of 16 tokens and more, so that keys 0..15 and 16..31 of a unit lie in
// one page each and their addresses are uniform but for a lane's constant offset.
template <class T, int D, int RT, bool WIDE>
__device__ __forceinline__ void attend_rows(const AttnArgs& a, const RowsPlan& plan, int block,
                                            char* lds) {
  constexpr int KC = D / 32;   // 32-element chunks of a key
  constexpr int DL = D / 16;   // elements of a value per lane
  constexpr int VW = DL / 2;   // dwords of them
  using elem = typename T::elem;
  using x8 = typename T::x8;
  const int lane = threadIdx.x & 63;
  const int col = lane & 15, h = lane >> 4;
  const int shift = a.kv.page_shift, page_mask = (1 << shift) - 1;
  auto dims_of = [](int c) { return (c >> 1) * 64 + (c & 1) * 8; };

  const RowsLine line = rows_line(a, plan, 16 * RT, block, lds);
  if (line.me >= line.waves) return;
  for (int64_t w = line.begin; w < line.end;) {
    const RowsPart part = rows_part(a, line, w);
    const int kh = part.kh, r = part.r, u0 = part.u0, u1 = part.u1;
    const Request x = request_of(a, r);
    const Span sp = rows_span(a, x);
    const int rows = rows_of(a, x);
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
                        (int64_t)qh * a.q_head + h * 16;
#pragma unroll
      for (int c = 0; c < KC; ++c) q[t][c] = *(const x8*)(src + dims_of(c));
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
    // byte offsets within a page fit 32 bits, and pages are counted in 16-byte pieces
    const char* kbase = (const char*)((const elem*)a.kv.k + kh * a.kv.k_head);
    const char* vbase = (const char*)((const elem*)a.kv.v + kh * a.kv.v_head);
    const uint32_t k_slot = (uint32_t)a.kv.k_slot * 2, v_slot = (uint32_t)a.kv.v_slot * 2;
    // Key s0 + (lane mod 32) of a unit: whether some row sees it, and its page.  The
    // page is read a unit ahead and looked at only when its turn comes.
    auto key_at = [&](int u) { return sp.block(u) * UNIT + (lane & 31); };
    auto seen = [&](int s) {
      return s < n_keys && (a.window == 0 || s > first_own - a.window || s < sink_keys);
    };
    auto page_at = [&](int u) {
      const int s = key_at(u);
      return table[seen(s) ? s >> shift : 0];
    };

    const int last = sp.blocks > 0 ? u1 : u0;  // a tile without keys has one unit, but no block
    int next = last > u0 ? page_at(u0) : 0;
    for (int u = u0; u < last; ++u) {
      const int s0 = sp.block(u) * UNIT;
      const int page = next;
      if (u + 1 < last) next = page_at(u + 1);
      const uint64_t found =
          __ballot(seen(key_at(u)) && (uint32_t)page < (uint32_t)a.kv.n_pages);
      if (found == 0) continue;
      // all 32 keys held, and seen by every row
      const bool full = found == ~0ull && s0 + UNIT - 1 <= first_own &&
                        (a.window == 0 || s0 > last_own - a.window ||
                         s0 + UNIT <= sink_keys);

      // where the keys that this lane loads lie; those that are not there read page 0 (the
      // cache has one, since some key was found) and are masked
      const char* ks[2];
      const char* vs[8];
      if constexpr (WIDE) {
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          const uint32_t half = (uint32_t)(found >> (b * 16)) & 0xffff;  // one page, if any
          const int pg =
              half ? __builtin_amdgcn_readlane(page, b * 16 + __builtin_ctz(half)) : 0;
          const uint32_t slot = (uint32_t)(s0 + b * 16) & page_mask;
          ks[b] = kbase + (uint64_t)(uint32_t)pg * (a.kv.k_page * 2) + (uint64_t)slot * k_slot;
          const char* v0 =
              vbase + (uint64_t)(uint32_t)pg * (a.kv.v_page * 2) + (uint64_t)slot * v_slot;
#pragma unroll
          for (int j = 0; j < 4; ++j) vs[b * 4 + j] = v0 + (uint64_t)j * v_slot;
        }
      } else {
        const int safe = (found >> lane) & 1 ? page : 0;
        int kp[2], vp[8];
#pragma unroll
        for (int b = 0; b < 2; ++b) kp[b] = __shfl(safe, b * 16 + col);
#pragma unroll
        for (int j = 0; j < 8; ++j) vp[j] = __shfl(safe, (j & 3) + 4 * h + (j >> 2) * 16);
#pragma unroll
        for (int b = 0; b < 2; ++b)
          ks[b] = kbase + (uint64_t)(uint32_t)kp[b] * (uint64_t)(a.kv.k_page * 2) +
                  (uint32_t)((s0 + b * 16 + col) & page_mask) * k_slot;
#pragma unroll
        for (int j = 0; j < 8; ++j)
          vs[j] = vbase + (uint64_t)(uint32_t)vp[j] * (uint64_t)(a.kv.v_page * 2) +
                  (uint32_t)((s0 + (j & 3) + 4 * h + (j >> 2) * 16) & page_mask) * v_slot;
      }
      const uint32_t k_lane = (WIDE ? col * k_slot : 0) + h * 32;
      const uint32_t v_lane = (WIDE ? 4 * h * v_slot : 0) + col * (DL * 2);
      x8 k[2][KC];
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int c = 0; c < KC; ++c)
          k[b][c] = __builtin_nontemporal_load((const x8*)(ks[b] + k_lane + dims_of(c) * 2));
      uint32_t v[8][VW];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if constexpr (VW == 2) {
          const u32x2 y = __builtin_nontemporal_load((const u32x2*)(vs[j] + v_lane));
          v[j][0] = y[0];
          v[j][1] = y[1];
        } else {
#pragma unroll
          for (int i = 0; i < VW; i += 4) {
            const u32x4 y = __builtin_nontemporal_load((const u32x4*)(vs[j] + v_lane + 4 * i));
#pragma unroll
            for (int e = 0; e < 4; ++e) v[j][i + e] = y[e];
          }
        }
      }

      // all of the unit's loads are under way before the first is waited for (left to
      // itself the scheduler puts the values' loads behind the first products)
      __builtin_amdgcn_sched_barrier(0);

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
          p[t][j] = (elem)e[j];  // the second product's operand (attend_common.hpp)
        }
      }

      if (found != ~0ull) {  // what sits where no key is may be anything: 0 * NaN would be NaN
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (!((found >> ((j & 3) + 4 * h + (j >> 2) * 16)) & 1)) {
#pragma unroll
            for (int i = 0; i < VW; ++i) v[j][i] = 0;
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

    rows_write<T, D, RT>(a, plan, line, part, w, x, rows, o, mu, l);
    w += u1 - u0;
  }
}

inline size_t rows_lds(int n_req) { return (size_t)(ATT_WAVES + n_req + 1) * sizeof(int64_t); }

}  // namespace fs
