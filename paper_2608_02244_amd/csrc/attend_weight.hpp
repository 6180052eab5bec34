// Attention weight of held tokens (fsched_attend_weight, fsched_attend4_weight):
//   weight[r][j] += sum over the new tokens i of request r and the query heads h that see
//   key j of exp(scale q_ih . k_j - lse_ih)
//
// S^T = K Q^T: a lane holds some keys of one row, whose lse is its own number; each key's
// sum over rows stays in its place through all rows and heads and is exchanged between
// lanes once at the end.  A key that is not there needs no mask: its sum is not written.
//   rows kernel   requests with few rows (tokens times query heads per key head): a wave
//     takes units of 32 keys, all key heads of each, keys straight from the cache into
//     registers, the next head's under way; bound by the bytes of the keys
//   tiles kernel  requests with many rows: a block holds 256 keys of a key head (128 with
//     heads of 256) in registers and goes over the rows that see them, which its waves share
//     through LDS; bound by the products and the exponentials
// In both the work of all requests forms one line, cut into equal pieces.  The rows kernel's
// pieces are whole keys, so that a key is one wave's; the tiles kernel's may cut a tile's
// rows, whose sums are then joined, in their order, by a second launch.  Equal calls give
// equal bits.
//
// Measured (heads of 128, bf16): 64 requests holding 65,000 tokens, 31 us or 4.3 TB/s; 512
// holding 0.73 M in 4 bits, 59 us or 3.5 TB/s (4.1 without the start); prompts of 25,600
// tokens, calls of 360 to 381 us on the cards that it ran on, 6 of them the joins and 5 a rows
// kernel that finds no request (the tiles alone 366 us or 820 TFLOP/s, traced on a card whose
// calls took 381); over 4 bits 350 us.
//
// Sums are of 32 bits.  A lane of the tiles kernel adds a key's terms one after the other, some
// 2,500 in those prompts, which errs by a root of their number: the weights are 1.6e-7 (of their
// norm) from 64 bits, and 8.7e-8 where terms are added pairwise.  Of decode steps both are
// 2.9e-8.
#pragma once
#include <hip/hip_runtime.h>

#include "attend_common.hpp"
#include "attend_tiles.hpp"
#include "fp4.hpp"

namespace fs {

constexpr float LOG2E = 1.4426950408889634f;
constexpr int WEIGHT_FEW = 32;   // rows of the rows kernel's requests, at most
constexpr int WEIGHT_UNIT = 32;  // keys of its units

__device__ __forceinline__ int weight_rows(const AttnArgs& a, int q_len) {
  return min(q_len, a.max_q) * a.group;
}

// Inclusive sums over n numbers in LDS, x[i] to the sum of those before it, x[n] to all.
__device__ __forceinline__ void sums_before(int64_t* x, int n, int64_t* wave_sum) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int per = (n + ATT_THREADS - 1) / ATT_THREADS;
  const int r0 = min(n, tid * per), r1 = min(n, r0 + per);
  int64_t sum = 0;
  for (int r = r0; r < r1; ++r) sum += x[r];
  int64_t s = sum;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int64_t y = __shfl_up(s, d);
    if (lane >= d) s += y;
  }
  if (lane == 63) wave_sum[wave] = s;
  __syncthreads();
  for (int w = 0; w < wave; ++w) s += wave_sum[w];
  int64_t at = s - sum;
  for (int r = r0; r < r1; ++r) {
    const int64_t y = x[r];
    x[r] = at;
    at += y;
  }
  if (tid == ATT_THREADS - 1) x[n] = at;
  __syncthreads();
}

// The request that unit w is of.
__device__ __forceinline__ int request_at(const int64_t* before, int n, int64_t w) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (before[mid] <= w) lo = mid;
    else hi = mid;
  }
  return uni_int(lo);
}

// Sum over the 16 lanes of a row of the wave.
__device__ __forceinline__ float sum_row16(float x) {
  auto turn = [&](auto c) {
    const int y = __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x),
                                              0x120 + decltype(c)::value, 0xf, 0xf, true);
    x += __builtin_bit_cast(float, y);
  };
  turn(Const<8>{});
  turn(Const<4>{});
  turn(Const<2>{});
  turn(Const<1>{});
  return x;
}

// ---------------------------------------------------------------- few rows

// A lane's share (D/4 elements) of one key, as loaded, of two groups of 16 keys.
template <int D, bool FP4>
struct WeightKeys {
  static constexpr int WORDS = FP4 ? D / 32 : D / 8;
  uint32_t w[2][WORDS];
  uint32_t scale[2];
};

// Blocks per compute unit, as many as the registers leave.  With 2 / 3 / 4: the heavy decode
// batch in 4 bits 79 / - / 57 us, 64 requests in 16 bits 37 / 32 / -.
constexpr int weight_occupancy(int D, int RT, bool fp4) {
  return D == 256 ? (RT == 2 ? 1 : 2) : RT == 2 ? (D == 64 ? 3 : 2) : fp4 || D == 64 ? 4 : 3;
}

template <class T, int D, int RT, int KIND>
__global__ __launch_bounds__(ATT_THREADS, weight_occupancy(D, RT, KIND == FP4_PAGES)) void
weight_rows_kernel(WeightArgs wa) {
  constexpr bool FP4 = KIND == FP4_PAGES, WIDE = KIND != SMALL_PAGES;
  constexpr int KC = D / 32;
  using elem = typename T::elem;
  using x8 = typename T::x8;
  using Keys = WeightKeys<D, FP4>;
  using G = Group4<D>;
  const AttnArgs& a = wa.at;
  extern __shared__ __attribute__((aligned(16))) char lds[];
  int64_t* wave_sum = (int64_t*)lds;       // [ATT_WAVES]
  int64_t* before = wave_sum + ATT_WAVES;  // [n_req + 1] units before request r
  __shared__ float shared_sum[ATT_WAVES][WEIGHT_UNIT];
  const int tid = threadIdx.x, lane = tid & 63, wave = uni_int(tid >> 6);
  const int col = lane & 15, h = lane >> 4;
  const int shift = a.kv.page_shift, page_mask = (1 << shift) - 1;

  auto span = [&](const Request& x) {
    const int p0 = x.kv - x.q_len, n = min(x.q_len, a.max_q);
    return span_of<WEIGHT_UNIT>(p0, p0 + n - 1, x.kv, a.window, a.n_sink, a.prefix_len);
  };
  for (int r = tid; r < a.n_req; r += ATT_THREADS) {
    const Request x = request_of(a, r);
    const int rows = weight_rows(a, x.q_len);
    before[r] = rows > 0 && rows <= 16 * RT ? span(x).blocks : 0;
  }
  __syncthreads();
  sums_before(before, a.n_req, wave_sum);
  const int64_t total = before[a.n_req];
  // Where there are fewer units than half or a quarter of the waves, two or four waves of a
  // block share a unit's key heads.
  const int64_t waves = (int64_t)gridDim.x * ATT_WAVES;
  const int heads = a.kv.kv_heads;  // (each share has one at least)
  const int shares = 4 * total <= waves && heads >= 4 ? 4 : 2 * total <= waves && heads >= 2 ? 2 : 1;
  const int64_t me = (int64_t)blockIdx.x * ATT_WAVES + wave, mine = me / shares;
  const int share = (int)(me % shares);
  int64_t begin = mine, end = min(mine + 1, total);
  if (shares == 1) {
    begin = total * me / waves;
    end = total * (me + 1) / waves;
  }
  const int kh0 = a.kv.kv_heads * share / shares, kh1 = a.kv.kv_heads * (share + 1) / shares;
  const int64_t k_head = a.kv.k_head * (FP4 ? 1 : 2);

  float* out = nullptr;  // of the lane's key of the last unit, if it has one
  float value = 0.0f;
  for (int64_t w = begin; w < end;) {
    const int r = request_at(before, a.n_req, w);
    const Request x = request_of(a, r);
    const Span sp = span(x);
    const int u0 = (int)(w - before[r]), u1 = (int)(min(end, before[r + 1]) - before[r]);
    w += u1 - u0;
    const int first_own = x.kv - x.q_len, n_new = min(x.q_len, a.max_q);
    const int last_own = first_own + n_new - 1, n_keys = min(x.kv, last_own + 1);
    const int sink_keys = a.window > 0 ? a.n_sink - a.prefix_len : 0;
    const int rows = n_new * a.group;
    const int32_t* table = a.table + (int64_t)r * a.width;

    // this lane's rows
    const elem* q_at[RT];
    const float* lse_at[RT];
    int top[RT], low[RT];
    bool on[RT];
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      const int row = t * 16 + col;
      on[t] = row < rows;
      const int tok = (on[t] ? row : 0) / a.group, g = on[t] ? row - tok * a.group : 0;
      q_at[t] = (const elem*)a.q + (int64_t)(x.q0 + tok) * a.q_token + (int64_t)g * a.q_head +
                (FP4 ? h * (D / 4) : h * 16);
      lse_at[t] = wa.lse + (int64_t)(x.q0 + tok) * a.q_heads + g;
      top[t] = on[t] ? first_own + tok : -1;
      low[t] = a.window > 0 ? top[t] - a.window : -0x7fffffff - 1;
    }
    auto seen = [&](int key) {
      return key < n_keys && (a.window == 0 || key > first_own - a.window || key < sink_keys);
    };
    // Pages of a unit's keys: of the lane's own key of each group, or of the whole group.
    auto pages_of = [&](int u, int (&pages)[2]) {
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const int j = sp.block(u) * WEIGHT_UNIT + b * 16, key = WIDE ? j : j + col;
        // a group has a key that is seen if its last one in the window's sense is
        const bool any = WIDE ? j < n_keys && (a.window == 0 || j + 15 > first_own - a.window ||
                                               j < sink_keys)
                              : seen(key);
        pages[b] = any ? table[key >> shift] : -1;
      }
    };
    // Where the lane's two keys of a unit lie (key head 0); those that are not there read
    // page 0.
    auto places = [&](int u, const int (&pages)[2], const char* (&at)[2]) {
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const int j = sp.block(u) * WEIGHT_UNIT + b * 16;
        const int page = WIDE ? uni_int(pages[b]) : pages[b];
        const uint32_t pg = (uint32_t)page < (uint32_t)a.kv.n_pages ? page : 0;
        if constexpr (FP4) {
          at[b] = (const char*)a.kv.k + pg * (uint64_t)a.kv.k_page +
                  ((j & page_mask) >> GROUP_SHIFT) * (uint64_t)a.kv.k_slot;
        } else {
          const int slot = (WIDE ? j : j + col) & page_mask;
          at[b] = (const char*)a.kv.k +
                  (pg * (uint64_t)a.kv.k_page + slot * (uint64_t)a.kv.k_slot) * 2;
        }
      }
    };
    const uint32_t lane_at = FP4 ? G::key(col) + h * (D / 8)
                                 : (WIDE ? col * (uint32_t)a.kv.k_slot * 2 : 0) + h * 32;
    const uint32_t scale_at = G::key_scale(col, h * (D / 4) / 32);
    auto load = [&](const char* const (&at)[2], int kh) {
      Keys k;
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const char* p = at[b] + kh * k_head;
        if constexpr (FP4) {
#pragma unroll
          for (int i = 0; i < Keys::WORDS; ++i)
            k.w[b][i] = __builtin_nontemporal_load((const uint32_t*)(p + lane_at) + i);
          k.scale[b] = D == 256 ? *(const uint16_t*)(p + scale_at)
                                : *(const uint8_t*)(p + scale_at);
        } else {
#pragma unroll
          for (int c = 0; c < KC; ++c) {
            const u32x4 y = __builtin_nontemporal_load(
                (const u32x4*)(p + lane_at + ((c >> 1) * 64 + (c & 1) * 8) * 2));
#pragma unroll
            for (int i = 0; i < 4; ++i) k.w[b][c * 4 + i] = y[i];
          }
        }
      }
      return k;
    };
    struct Item {  // a unit and a key head, heads first
      Keys k;
      x8 q[RT][KC];
      float lse[RT];
    };
    // Two items are under way while one is worked on: its place is loaded again as soon as
    // the products have read it.
    int pages[2], later[2], fetch_u = u0, fetch_kh = kh0;
    const char* at[2];
    pages_of(u0, pages);
    places(u0, pages, at);
    if (u0 + 1 < u1) pages_of(u0 + 1, later);
    auto fetch = [&](Item& y) {
      if (fetch_u >= u1) return;
      y.k = load(at, fetch_kh);
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        const elem* src = q_at[t] + (int64_t)fetch_kh * a.group * a.q_head;
#pragma unroll
        for (int c = 0; c < KC; ++c)
          y.q[t][c] = *(const x8*)(src + (FP4 ? c * 8 : (c >> 1) * 64 + (c & 1) * 8));
        y.lse[t] = lse_at[t][fetch_kh * a.group];
      }
      if (++fetch_kh == kh1) {
        fetch_kh = kh0;
        if (++fetch_u < u1) {
          places(fetch_u, later, at);
          if (fetch_u + 1 < u1) pages_of(fetch_u + 1, later);
        }
      }
    };
    int u = u0, kh = kh0, here[2];
    float sum[2][4] = {};
    // lane `col` < 8 of each row of lanes has key 16 (col / 4) + 4h + col mod 4 of a unit
    const int j = (col >> 2) * 16 + 4 * h + (col & 3);
    float old = 0.0f;
    auto begin_unit = [&]() {  // its pages and old weights, for the write behind its last head
      pages_of(u, here);
      const int key = sp.block(u) * WEIGHT_UNIT + j;
      old = 0.0f;
      if (col < 8 && seen(key)) old = wa.weight[(int64_t)r * wa.weight_stride + key];
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[b][e] = 0.0f;
    };
    auto work = [&](Item& now) {
      const int s0 = sp.block(u) * WEIGHT_UNIT;
      const bool full = s0 + WEIGHT_UNIT - 1 <= first_own &&
                        (a.window == 0 || s0 > last_own - a.window ||
                         s0 + WEIGHT_UNIT <= sink_keys);
      x8 k[2][KC];
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int c = 0; c < KC; ++c) {
          if constexpr (FP4) {
            const uint32_t byte = D == 256 ? (now.k.scale[b] >> (c / 4 * 8)) & 255 : now.k.scale[b];
            k[b][c] = __builtin_bit_cast(x8, values8<T>(now.k.w[b][c], scale_of(byte)));
          } else {
            k[b][c] = __builtin_bit_cast(x8, (u32x4){now.k.w[b][4 * c], now.k.w[b][4 * c + 1],
                                                     now.k.w[b][4 * c + 2], now.k.w[b][4 * c + 3]});
          }
        }
      f32x4 s[RT][2];
      float lse[RT];
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        lse[t] = now.lse[t];
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          s[t][b] = (f32x4){0, 0, 0, 0};
#pragma unroll
          for (int c = 0; c < KC; ++c) s[t][b] = T::mfma16(k[b][c], now.q[t][c], s[t][b]);
        }
      }
      fetch(now);
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        // a row that sees nothing, or is none, gives nothing
        const bool some = on[t] && lse[t] != NEG_INF;
        const float off = lse[t] * LOG2E;
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float p = exp2_fast(fmaf(s[t][b][e], a.scale_log2, -off));
            const int key = s0 + b * 16 + 4 * h + e;
            const bool see =
                some && (full || (key <= top[t] && (key > low[t] || key < sink_keys)));
            sum[b][e] += see ? p : 0.0f;
          }
      }
      if (++kh < kh1) return;
      kh = kh0;
      float v = 0.0f;
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float y = sum_row16(sum[b][e]);
          v = col == b * 4 + e ? y : v;
        }
      const int key = s0 + j;
      int page = col < 4 ? here[0] : here[1];
      if constexpr (!WIDE) {  // the lane that looked this key up
        const int p0 = __shfl(here[0], j & 15), p1 = __shfl(here[1], j & 15);
        page = col < 4 ? p0 : p1;
      }
      const bool writes = col < 8 && seen(key) && (uint32_t)page < (uint32_t)a.kv.n_pages;
      out = writes ? wa.weight + (int64_t)r * wa.weight_stride + key : nullptr;
      value = v;
      if (shares == 1 && out) *out = old + v;
      if (shares > 1 && col < 8) shared_sum[wave][j] = v;
      if (++u < u1) begin_unit();
    };
    Item ring[2];
    fetch(ring[0]);
    fetch(ring[1]);
    begin_unit();
    while (u < u1) {
      work(ring[0]);
      if (u < u1) work(ring[1]);
    }
  }
  if (shares == 1) return;
  __syncthreads();  // all threads of the block: `shares` is the same for the launch
  if (share == 0 && out) {
    const int j = (col >> 2) * 16 + 4 * h + (col & 3);
    for (int i = 1; i < shares; ++i) value += shared_sum[wave + i][j];
    *out += value;
  }
}

// --------------------------------------------------------------- many rows

// 4 bytes per lane from src + off to LDS at base + 4 * lane, as load_to_lds does.
__device__ __forceinline__ void load_dword_to_lds(const char* src, uint32_t off, uint32_t base) {
  uint32_t m0;
  asm volatile(
      "s_mov_b32 %0, m0\n\t"
      "s_mov_b32 m0, %3\n\t"
      "s_nop 0\n\t"
      "global_load_lds_dword %1, %2\n\t"
      "s_mov_b32 m0, %0"
      : "=&s"(m0)
      : "v"(off), "s"(src), "s"(base)
      : "memory");
}

// All loads but the last N.
template <int N>
__device__ __forceinline__ void wait_loads_but() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

// What a tile and key head takes beside its stages (keys to load, the first rows to wait
// for), in stages.  Prompts of 25,600 tokens with 0 / 4 / 8 / 12: 410 /
// 390 / 384 / 386 us.
constexpr int WEIGHT_START = 8;

// A part of a tile that a later block goes on with: written by the block that begins it.
struct WeightTile {
  int32_t r, key;  // request, first key
  int32_t first;   // slot of the first part; the next blocks' first slots follow
  int32_t count;   // parts, 0: none
};

struct WeightPlan {
  int32_t blocks;
  float* part;        // [2 blocks][keys of a tile]
  WeightTile* tiles;  // [blocks]
};

template <int D>
struct WeightTileOf {
  static constexpr int GROUPS = D == 256 ? 1 : 2;        // of 32 keys, of a wave
  static constexpr int KEYS = GROUPS * 32 * ATT_WAVES;   // of a tile
  static constexpr int ROWS = 64;                        // of a stage
  static constexpr int PIECES = D / 8;                   // 16-byte pieces of a row
  static constexpr int LOADS = ROWS * PIECES / ATT_THREADS;
  static constexpr int BYTES = ROWS * D * 2;
  static constexpr int BUFFERS = D == 256 ? 2 : 3;       // stages in LDS, one being read
  static constexpr int LDS = BUFFERS * (BYTES + 256);    // and the line's sums
};

// Registers: heads of 128 take all 256 and spill 22 (26 over 4 bits).  Those are the thread's
// rows of a stage, which `fetch` reads back, each behind a wait for all loads, where it makes the
// offsets anew: at a tile's start and end, and in every stage where 64 is no multiple of the
// group.  The stages under way are waited for with them: prompts with 5 query heads to a key
// head take 493 us, 10 % more for each product than with 4.  Counted in the prompts with 4:
// vector instructions issue in 54 % of the cycles, the matrix units are busy in 36 %, and 1.6 of
// 2 waves are there.
template <class T, int D, bool FP4>
__global__ __launch_bounds__(ATT_THREADS, 2) void weight_tiles_kernel(WeightArgs wa,
                                                                      WeightPlan plan) {
  using L = WeightTileOf<D>;
  constexpr int NK = L::GROUPS, KB = L::KEYS, SR = L::ROWS, QC = D / 16, TILES = SR / 32;
  using elem = typename T::elem;
  using x8 = typename T::x8;
  using G = Group4<D>;
  const AttnArgs& a = wa.at;
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  // LDS: NB stages of rows, their rows' lse, the line's sums
  constexpr int NB = L::BUFFERS;
  const float* lse_in = (const float*)(lds + NB * L::BYTES);             // [NB][64]
  int64_t* wave_sum = (int64_t*)(lds + L::LDS);                          // [ATT_WAVES]
  int64_t* before = wave_sum + ATT_WAVES;              // [n_req + 1] units before request r
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds;
  const int tid = threadIdx.x, lane = tid & 63, wave = uni_int(tid >> 6);
  const int col = lane & 31, h = lane >> 5;
  const int shift = a.kv.page_shift, page_mask = (1 << shift) - 1;
  const int sink_keys = a.window > 0 ? a.n_sink - a.prefix_len : 0;

  struct Shape {  // a request's tiles and rows
    int first_own, n_new, n_keys;
    Span sp;
  };
  auto shape_of = [&](int q_len, int kv) {
    Shape s;
    s.first_own = kv - q_len;
    s.n_new = min(q_len, a.max_q);
    const int last_own = s.first_own + s.n_new - 1;
    s.n_keys = min(kv, last_own + 1);
    s.sp = span_of<KB>(s.first_own, last_own, kv, a.window, a.n_sink, a.prefix_len);
    return s;
  };
  // rows of tile i that see some key of it: first .. last - 1
  struct RowsOf {
    int first, last;
  };
  auto rows_of_tile = [&](const Shape& s, int i) {
    const int k0 = s.sp.block(i) * KB, k1 = min(k0 + KB, s.n_keys);
    int from = max(0, k0 - s.first_own), to = s.n_new;
    if (a.window > 0 && k0 >= sink_keys)
      to = (int)max((int64_t)0, min((int64_t)to, (int64_t)k1 - 1 + a.window - s.first_own));
    return RowsOf{from * a.group, max(from, to) * a.group};
  };
  auto stages_of = [&](const Shape& s, int i) {
    const RowsOf y = rows_of_tile(s, i);
    return (y.last - y.first + SR - 1) / SR;
  };
  // units of a tile and key head: its stages, and what it takes to begin them
  auto units_of = [&](const Shape& s, int i) {
    const int n = stages_of(s, i);
    return n > 0 ? n + WEIGHT_START : 0;
  };
  // units of every request: its lengths first
  for (int r = tid; r < a.n_req; r += ATT_THREADS) {
    const Request x = request_of(a, r);
    const bool many = weight_rows(a, x.q_len) > WEIGHT_FEW;
    before[r] = many ? (int64_t)x.q_len << 32 | (uint32_t)x.kv : 0;
  }
  __syncthreads();
  for (int r = wave; r < a.n_req; r += ATT_WAVES) {
    const int64_t packed = before[r];
    if (packed == 0) continue;
    const Shape s = shape_of((int)(packed >> 32), (int)(uint32_t)packed);
    int64_t sum = 0;
    for (int i = lane; i < s.sp.blocks; i += 64) sum += units_of(s, i);
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) sum += __shfl_xor(sum, d);
    if (lane == 0) before[r] = sum * a.kv.kv_heads;
  }
  __syncthreads();
  sums_before(before, a.n_req, wave_sum);
  const int64_t total = before[a.n_req];
  // blocks with work: none has an empty piece, so a tile's parts are of consecutive blocks
  const int64_t blocks = min((int64_t)plan.blocks, total), me = blockIdx.x;
  const int64_t begin = me < blocks ? total * me / blocks : 0;
  const int64_t end = me < blocks ? total * (me + 1) / blocks : 0;
  auto block_of = [&](int64_t unit) {  // the block whose piece has it
    return (int)(((unit + 1) * blocks - 1) / total);
  };
  if (tid == 0) plan.tiles[blockIdx.x].count = 0;

  const int f = Tile<D>::swizzle(col);
  for (int64_t w = begin; w < end;) {
    const int r = request_at(before, a.n_req, w);
    const Request x = request_of(a, r);
    const Shape s = shape_of(x.q_len, x.kv);
    // which tile: 64 at a time
    int64_t rest = w - before[r];
    int tile = 0, head_units = 0;
    for (int i0 = 0;; i0 += 64) {
      const int n = i0 + lane < s.sp.blocks ? units_of(s, i0 + lane) : 0;
      int64_t sum = (int64_t)n * a.kv.kv_heads;
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) {
        const int64_t y = __shfl_up(sum, d);
        if (lane >= d) sum += y;
      }
      const uint64_t past = __ballot(sum > rest);
      if (past) {
        const int l = __builtin_ctzll(past);
        tile = i0 + l;
        head_units = __builtin_amdgcn_readlane(n, l);
        rest -= (int64_t)lane_of((uint64_t)sum, l) - (int64_t)head_units * a.kv.kv_heads;
        break;
      }
      rest -= (int64_t)lane_of((uint64_t)sum, 63);
      if (i0 + 64 >= s.sp.blocks) return;  // cannot be: the unit is one of the request's
    }
    const int64_t units = (int64_t)head_units * a.kv.kv_heads;
    const int64_t u0 = rest, u1 = min(units, u0 + (end - w));
    const RowsOf span_rows = rows_of_tile(s, tile);
    const int key0 = s.sp.block(tile) * KB;
    const int32_t* table = a.table + (int64_t)r * a.width;

    // the lane's keys (as the first operand's rows): where they lie
    // 32 keys from group_key[n] on: with two groups those at equal distance from both ends, so
    // that the waves share a tile's upper right corner (keys past the rows') evenly
    int group_key[NK];
#pragma unroll
    for (int n = 0; n < NK; ++n)
      group_key[n] = key0 + 32 * (n == 0 ? wave : 2 * ATT_WAVES - 1 - wave);
    const char* key_at[NK];
    uint32_t scale_at[NK];
#pragma unroll
    for (int n = 0; n < NK; ++n) {
      const int key = group_key[n] + col;
      const bool see = key < s.n_keys && (a.window == 0 || key > s.first_own - a.window ||
                                          key < sink_keys);
      const int page = see ? table[key >> shift] : -1;
      const uint32_t pg = (uint32_t)page < (uint32_t)a.kv.n_pages ? page : 0;
      const int slot = key & page_mask;
      if constexpr (FP4) {
        const int t = slot & (GROUP - 1);
        key_at[n] = (const char*)a.kv.k + pg * (uint64_t)a.kv.k_page +
                    (slot >> GROUP_SHIFT) * (uint64_t)a.kv.k_slot + G::key(t) + h * (D / 4);
        scale_at[n] = G::key_scale(t, 0) - G::key(t) - h * (D / 4) + h * (D / 64);
      } else {
        key_at[n] = (const char*)((const elem*)a.kv.k + pg * (uint64_t)a.kv.k_page +
                                  slot * (uint64_t)a.kv.k_slot + h * (D / 2));
        scale_at[n] = 0;
      }
    }
    float sum[NK][16];
#pragma unroll
    for (int n = 0; n < NK; ++n)
#pragma unroll
      for (int i = 0; i < 16; ++i) sum[n][i] = 0.0f;

    for (int64_t u = u0; u < u1;) {
      const int kh = (int)(u / head_units), i0 = (int)(u % head_units);
      const int i1 = (int)min((int64_t)head_units, i0 + (u1 - u));
      u += i1 - i0;
      const int st0 = max(0, i0 - WEIGHT_START), st1 = max(0, i1 - WEIGHT_START);
      if (st0 >= st1) continue;
      // Rows of a stage are fetched from a uniform base (its first row's token) and 32-bit
      // offsets of the thread, which stay the same where SR rows are whole tokens.  Rows past
      // the last one are read as that; their lse beside them, every wave the same.
      const char* q_of = (const char*)((const elem*)a.q + (int64_t)x.q0 * a.q_token +
                                       (int64_t)kh * a.group * a.q_head);
      const char* lse_of = (const char*)(wa.lse + (int64_t)x.q0 * a.q_heads + kh * a.group);
      const uint32_t q_token = (uint32_t)a.q_token * 2, q_head = (uint32_t)a.q_head * 2;
      const bool whole_tokens = SR % a.group == 0;
      uint32_t q_off[L::LOADS], lse_off = 0;
      int next_fetch = st0;
      auto fetch = [&](int buf) {
        const int r0 = span_rows.first + next_fetch * SR;
        const int tok0 = wa.group.divide(r0);
        if (next_fetch == st0 || !whole_tokens || r0 + SR > span_rows.last) {
          auto at = [&](int in_stage, uint32_t token, uint32_t head) {
            const int n = min(r0 + in_stage, span_rows.last - 1) - tok0 * a.group;
            const int t = wa.group.divide(n);
            return (uint32_t)t * token + (uint32_t)(n - t * a.group) * head;
          };
#pragma unroll
          for (int i = 0; i < L::LOADS; ++i) {
            const int in_stage = i * (ATT_THREADS / L::PIECES) + tid / L::PIECES;
            q_off[i] = at(in_stage, q_token, q_head) +
                       ((tid % L::PIECES) ^ Tile<D>::swizzle(in_stage)) * 16;
          }
          lse_off = at(lane, a.q_heads * 4, 4);
        }
        load_dword_to_lds(lse_of + (int64_t)tok0 * a.q_heads * 4, lse_off,
                          uni_int(lds0 + NB * L::BYTES + buf * 256));
        const char* base = q_of + (int64_t)tok0 * (a.q_token * 2);
#pragma unroll
        for (int i = 0; i < L::LOADS; ++i)
          load_to_lds(base, q_off[i],
                      uni_int(lds0 + buf * L::BYTES + (i * ATT_THREADS + wave * 64) * 16));
        ++next_fetch;
      };
      __syncthreads();  // the buffers are read
      fetch(0);
      if (NB == 3 && st0 + 1 < st1) fetch(1);
      x8 k[NK][QC];
#pragma unroll
      for (int n = 0; n < NK; ++n) {
        const char* p = key_at[n] + kh * (a.kv.k_head * (FP4 ? 1 : 2));
        if constexpr (FP4) {
          uint32_t words[QC];
#pragma unroll
          for (int c = 0; c < QC; ++c) words[c] = ((const uint32_t*)p)[c];
#pragma unroll
          for (int c = 0; c < QC; ++c) {
            const uint32_t byte = *(const uint8_t*)(p + (int32_t)scale_at[n] + c / 4);
            k[n][c] = __builtin_bit_cast(x8, values8<T>(words[c], scale_of(byte)));
          }
        } else {
#pragma unroll
          for (int c = 0; c < QC; ++c) k[n][c] = *(const x8*)(p + c * 16);
        }
      }
      // The keys are waited for here: left to itself the compiler waits in the loop below,
      // for the next stage's loads too.
#pragma unroll
      for (int n = 0; n < NK; ++n)
#pragma unroll
        for (int c = 0; c < QC; ++c) {
          u32x4 y = __builtin_bit_cast(u32x4, k[n][c]);
          asm volatile("" : "+v"(y));
          k[n][c] = __builtin_bit_cast(x8, y);
        }
      // Of a row tile: the lane's offset and last key, and whether its lse is NaN; the least
      // of all lanes' keys (-1: some lane is to be looked at) and the greatest.
      struct Rows {
        float off;
        int last, k0, k1;
        bool nan;
      };
      auto hide = [&](f32x16& x, int n, const Rows& y) {  // scores of keys that the row does not see
        if (group_key[n] + 31 <= y.k0 && (a.window == 0 || group_key[n] > y.k1 - a.window ||
                                          group_key[n] + 32 <= sink_keys))
          return;
        if (__ballot(y.nan)) {
#pragma unroll
          for (int i = 0; i < 16; ++i) x[i] = y.nan ? __builtin_nanf("") : x[i];
        }
        // against the lane's first key, so that the others are constants
        const int first = group_key[n] + 4 * h, top = y.last - first;
        if (a.window == 0) {
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (8 * (i / 4) + (i % 4) > top) x[i] = NEG_INF;
        } else {
          const int low = top - a.window, sinks = sink_keys - first;
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int key = 8 * (i / 4) + (i % 4);
            const bool see = (key <= top) & ((key > low) | (key < sinks));
            x[i] = see ? x[i] : NEG_INF;
          }
        }
      };
      auto add = [&](const f32x16& x, int n, const Rows& y) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          sum[n][i] += exp2_fast(fmaf(x[i], a.scale_log2, -y.off));
          asm volatile("" : "+v"(sum[n][i]));  // here, not wherever the sum is next looked at
        }
      };
      int buf = 0;
      for (int st = st0; st < st1; ++st) {
        // all but the loads of the stages behind this one
        if (NB == 3 && st + 1 < st1) wait_loads_but<L::LOADS + 1>();
        else wait_loads();
        __syncthreads();  // the stage is there; the buffer before it is free
        if (st + NB - 1 < st1) fetch(buf == 0 ? NB - 1 : buf - 1);
        // piece h QC + c of row `col`: c takes the low bits of the place only
        const uint32_t row_lds =
            lds0 + buf * L::BYTES + col * (D * 2) + ((h * QC) ^ f) * 16;
        u32x4 q[QC];
        auto read_row = [&](int t, int c) {
          q[c] = read16((row_lds ^ (c * 16)) + t * (32 * D * 2));
        };
#pragma unroll
        for (int c = 0; c < QC; ++c) read_row(0, c);
        Rows y[TILES];
#pragma unroll
        for (int t = 0; t < TILES; ++t) {
          const int row = span_rows.first + st * SR + t * 32 + col;
          const float l = lse_in[buf * 64 + t * 32 + col];
          y[t].last = s.first_own + wa.group.divide(min(row, span_rows.last - 1));
          y[t].off = l * LOG2E;
          y[t].nan = false;
          y[t].k0 = __builtin_amdgcn_readlane(y[t].last, 0);
          y[t].k1 = __builtin_amdgcn_readlane(y[t].last, 31);
          // A row that sees nothing, or is none, gives nothing whatever its scores are: all its
          // keys are hidden.  One whose lse is NaN gives that to the keys that it sees only.
          const bool none = row >= span_rows.last || l == NEG_INF;
          if (__ballot(none || l != l)) {
            y[t].last = none ? -1 : y[t].last;
            y[t].off = none || l != l ? 0.0f : y[t].off;
            y[t].nan = l != l;
            y[t].k0 = -1;
          }
        }
        // A step is a row tile and 32 keys.  Its exponentials are taken beside the products of
        // the next: two sets of scores in turn.
        f32x16 score[2];
        auto steps = [&](auto first, auto last) {  // over the groups of keys first .. last
          constexpr int N0 = decltype(first)::value, N1 = decltype(last)::value, N = N1 - N0 + 1;
#pragma unroll
          for (int j = 0; j < TILES * N; ++j) {
            const int t = j / N, n = N0 + j % N;
            const bool reads = n == N1 && t + 1 < TILES;  // the next row tile's operands
            if (j > 0) hide(score[(j - 1) & 1], N0 + (j - 1) % N, y[(j - 1) / N]);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < 16; ++i) score[j & 1][i] = 0.0f;
#pragma unroll
            for (int c = 0; c < QC; ++c) {
              score[j & 1] = T::mfma32(k[n][c], __builtin_bit_cast(x8, q[c]), score[j & 1]);
              if (reads) read_row(t + 1, c);
            }
            if (j > 0) add(score[(j - 1) & 1], N0 + (j - 1) % N, y[(j - 1) / N]);
            // the order: a few exponentials beside each product
#pragma unroll
            for (int c = 0; c < QC; ++c) {
              __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);                     // product
              if (j > 0) __builtin_amdgcn_sched_group_barrier(0x402, 48 / QC, 0);    // VALU
              if (reads) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);          // LDS read
            }
            __builtin_amdgcn_sched_barrier(0);
          }
          constexpr int J = TILES * N - 1;
          hide(score[J & 1], N1, y[TILES - 1]);
          add(score[J & 1], N1, y[TILES - 1]);
        };
        const int k1 = y[TILES - 1].k1;  // keys behind it are seen by none of the rows
        if constexpr (NK == 1) {
          if (group_key[0] <= k1) steps(Const<0>{}, Const<0>{});
        } else {
          // group 0 comes before group 1
          if (group_key[1] <= k1) steps(Const<0>{}, Const<1>{});
          else if (group_key[0] <= k1) steps(Const<0>{}, Const<0>{});
        }
        buf = buf + 1 == NB ? 0 : buf + 1;
      }
    }

    const bool whole = u0 == 0 && u1 == units;
    const int slot = 2 * (int)blockIdx.x + (w != begin);
    if (!whole && u0 == 0 && tid == 0)
      plan.tiles[blockIdx.x] = WeightTile{r, key0, slot, block_of(w + units - 1) -
                                                             (int)blockIdx.x + 1};
#pragma unroll
    for (int n = 0; n < NK; ++n) {
      float v = 0.0f;  // lane `col` < 16 has key 8 (col / 4) + 4h + col mod 4
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float y = sum_xor16(sum_row16(sum[n][i]));
        v = col == i ? y : v;
      }
      if (col >= 16) continue;
      const int at = group_key[n] - key0 + 8 * (col / 4) + 4 * h + col % 4;
      if (!whole) {
        plan.part[(int64_t)slot * KB + at] = v;
        continue;
      }
      const int key = key0 + at;
      if (key < s.n_keys && (a.window == 0 || key > s.first_own - a.window || key < sink_keys) &&
          (uint32_t)table[key >> shift] < (uint32_t)a.kv.n_pages)
        wa.weight[(int64_t)r * wa.weight_stride + key] += v;
    }
    w += u1 - u0;
  }
}

// Parts of tiles that several blocks worked on, joined in their order.
template <int KB>
__global__ __launch_bounds__(KB) void weight_join_kernel(WeightArgs wa, WeightPlan plan) {
  const AttnArgs& a = wa.at;
  const WeightTile t = plan.tiles[blockIdx.x];
  if (t.count == 0) return;
  const Request x = request_of(a, t.r);
  const int first_own = x.kv - x.q_len, last_own = first_own + min(x.q_len, a.max_q) - 1;
  const int n_keys = min(x.kv, last_own + 1), key = t.key + threadIdx.x;
  const int sink_keys = a.window > 0 ? a.n_sink - a.prefix_len : 0;
  if (key >= n_keys) return;
  if (a.window > 0 && key <= first_own - a.window && key >= sink_keys) return;
  const int page = a.table[(int64_t)t.r * a.width + (key >> a.kv.page_shift)];
  if ((uint32_t)page >= (uint32_t)a.kv.n_pages) return;
  float v = plan.part[(int64_t)t.first * KB + threadIdx.x];
  for (int i = 1; i < t.count; ++i)
    v += plan.part[2 * ((int64_t)blockIdx.x + i) * KB + threadIdx.x];
  wa.weight[(int64_t)t.r * wa.weight_stride + key] += v;
}

}  // namespace fs
