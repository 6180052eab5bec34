// Attention for many rows: prompts and chunks of them over what their request
// holds, and the rows of all tokens over a shared prefix.
//
// A block takes 128 rows (tokens times the query heads of one key head, 32 per
// wave) and goes over their keys in tiles, which its four waves share through
// LDS; the next tile arrives by direct loads while one is worked on.
//   S^T = K Q^T    32 keys x 32 rows, K rows from LDS, Q in registers
//   O^T = V^T P^T  the scores leave the first product with a lane holding, of its
//     row, keys 8g + 4h + 0..3 (h: half of the wave); the contraction takes them
//     in that order, so P stays in its lanes, and the transposing LDS loads bring
//     the values of those keys, one element of the head per lane.
// A 16-byte piece c of key j lies at piece c ^ f(j) of its row, f a permutation of
// the low bits that spreads both reads over all banks: the first takes one piece
// of 32 keys at once, the second 64 bytes of 8 keys.
//
// Bound by the products.  Measured (heads of 128, bf16): prompts of 25,600 tokens in all,
// 667 to 728 us a call (898 to 823 TFLOP/s) on the cards that it ran on, once some 25 calls
// have gone before; the first ten take 750 to 850, while the clock finds its level.  As
// launches among such first ones: reading the operands one step ahead of their products,
// uniform load addresses and clearing absent keys in LDS rather than in each operand took
// them from 985 to 800 us, masks without branches and lane-computed addresses from 790 to
// 757 us.
#pragma once
#include <hip/hip_runtime.h>

#include "attend_common.hpp"
#include "fp4.hpp"

namespace fs {

constexpr int TILE_ROWS = 128;  // rows of a block

struct TilesPlan {
  int32_t prefix;    // 1: rows of all tokens over the prefix's keys; 0: of each request over its own
  int32_t min_rows;  // own keys: requests with at most this many rows are another kernel's
  int32_t split;     // parts that a tile's keys are cut into
  int32_t parts;     // 1: write parts (always where split > 1)
  float* part_o;     // [split][n_tok * q_heads][head_dim]
  float2* part_ml;   // [split][n_tok * q_heads] (mu, l)
};

template <int D>
struct Tile {
  static constexpr int KEYS = D == 256 ? 32 : 64;
  static constexpr int PIECES = D / 8;                       // 16-byte pieces of a key
  static constexpr int LOADS = KEYS * PIECES / ATT_THREADS;      // direct loads per thread
  static constexpr int BYTES = KEYS * D * 2;
  static __device__ __forceinline__ int swizzle(int key) {
    return D == 64 ? (((key >> 1) & 1) << 2) | ((key >> 2) & 3)
                   : ((key & 3) << 2) | ((key >> 2) & 3);
  }
};

// 16 bytes per lane from global memory to LDS at base + 16 * lane.  The compiler
// does not count these; they are waited for by hand before the block's barrier.  (Loads
// that it counts it waits for before each read of LDS, the next tile's before this one's.)
// They take the LDS address from m0, which is the compiler's own: it is put back (prompts
// of 25,600 tokens 724 us a call without that, 728 with it).
__device__ __forceinline__ void load_to_lds(const void* src, uint32_t base) {
  uint32_t m0;
  asm volatile(
      "s_mov_b32 %0, m0\n\t"
      "s_mov_b32 m0, %2\n\t"
      "s_nop 0\n\t"
      "global_load_lds_dwordx4 %1, off\n\t"
      "s_mov_b32 m0, %0"
      : "=&s"(m0)
      : "v"(src), "s"(base)
      : "memory");
}

// The same from base + off, the base uniform.
__device__ __forceinline__ void load_to_lds(const char* src, uint32_t off, uint32_t base) {
  uint32_t m0;
  asm volatile(
      "s_mov_b32 %0, m0\n\t"
      "s_mov_b32 m0, %3\n\t"
      "s_nop 0\n\t"
      "global_load_lds_dwordx4 %1, %2\n\t"
      "s_mov_b32 m0, %0"
      : "=&s"(m0)
      : "v"(off), "s"(src), "s"(base)
      : "memory");
}

__device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

__device__ __forceinline__ u32x2 read_transposed(uint32_t addr) {
  return __builtin_bit_cast(
      u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(uintptr_t)addr));
}

__device__ __forceinline__ u32x4 read16(uint32_t addr) {
  return *(__attribute__((address_space(3))) u32x4*)(uintptr_t)addr;
}

__device__ __forceinline__ void write16(uint32_t addr, u32x4 v) {
  *(__attribute__((address_space(3))) u32x4*)(uintptr_t)addr = v;
}

__device__ __forceinline__ void write8(uint32_t addr, u32x2 v) {
  *(__attribute__((address_space(3))) u32x2*)(uintptr_t)addr = v;
}

__device__ __forceinline__ uint64_t lane_of(uint64_t x, int lane) {
  const uint32_t lo = __builtin_amdgcn_readlane((int)(uint32_t)x, lane);
  const uint32_t hi = __builtin_amdgcn_readlane((int)(uint32_t)(x >> 32), lane);
  return (uint64_t)hi << 32 | lo;
}

__device__ __forceinline__ uint64_t shuffled(uint64_t x, int lane) {
  const uint32_t lo = __shfl((int)(uint32_t)x, lane), hi = __shfl((int)(uint32_t)(x >> 32), lane);
  return (uint64_t)hi << 32 | lo;
}

// A thread's share of a tile in 4 bits: D / (256 / KEYS) elements of one key, and as many of
// the values (a piece's, of the four tokens of a quarter of a group, or half of it).
template <int D>
struct Tile4 {
  static constexpr int SHARE = ATT_THREADS / Tile<D>::KEYS;  // threads of a key
  static constexpr int WORDS = D / SHARE / 8;                // dwords of codes each side
  uint32_t k[WORDS], v[WORDS], k_scale, v_scale;             // scales as loaded
};

// KIND SMALL_PAGES, WIDE_PAGES (of 16 tokens and more: the keys that a wave loads at once,
// 8, 4 or 2 from a multiple of that on, then lie in one page, and their addresses are
// uniform but for a lane's constant offset) or FP4_PAGES (a cache of 4 bits: the tile goes
// through registers, where its codes become elements, into the same places in LDS; loaded
// two tiles ahead, converted one ahead: prompts of 25,600 tokens 691 us, as over 16 bits).
template <class T, int D, int KIND>
__device__ __forceinline__ void attend_tiles(const AttnArgs& a, const TilesPlan& plan, int block,
                                             char* lds) {
  using L = Tile<D>;
  constexpr bool WIDE = KIND == WIDE_PAGES, FP4 = KIND == FP4_PAGES;
  constexpr int KB = L::KEYS, NT = KB / 32, QC = D / 16, DT = D / 32;
  using elem = typename T::elem;
  using x8 = typename T::x8;
  // LDS: K and V of two tiles, then a few words
  int(*reduce)[ATT_WAVES] = (int(*)[ATT_WAVES])(lds + 4 * L::BYTES);  // [2]
  int* found_tile = reduce[2];                                        // [2]
  int* class_tiles = reduce[3];                                       // [8]
  int32_t* starts = (int32_t*)(lds + 4 * L::BYTES + 256);             // [n_req + 1], prefix only

  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int col = lane & 31, h = lane >> 5;
  const int shift = a.kv.page_shift, page_mask = (1 << shift) - 1;
  int id = block;
  const int kh = id % a.kv.kv_heads;
  id /= a.kv.kv_heads;
  const int part = id % plan.split;
  int tile = id / plan.split;

  const int offset = plan.prefix ? 0 : a.prefix_len;  // position of key 0
  const int sink_keys = a.window > 0 ? a.n_sink - offset : 0;
  const int32_t* table = a.prefix_pages;  // own keys: set once the request is known
  // The keys that the block's rows see: n_keys and tiles b0 .. b1 of span sp.
  int n_keys = 0, b0 = 0, b1 = 0, bmin = 0;
  Span sp = {0, 0, 0};
  auto cut = [&]() {
    b0 = (int)((int64_t)sp.blocks * part / plan.split);
    b1 = (int)((int64_t)sp.blocks * (part + 1) / plan.split);
  };
  // LDS places: buffer b holds K at 2 b BYTES, V behind it
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds;
  const char* kbase = (const char*)((const elem*)a.kv.k + kh * a.kv.k_head);
  const char* vbase = (const char*)((const elem*)a.kv.v + kh * a.kv.v_head);
  const uint32_t k_slot = (uint32_t)a.kv.k_slot * 2, v_slot = (uint32_t)a.kv.v_slot * 2;
  // Key (lane mod KB) of tile b: whether some row of the block sees it, and its page (for
  // keys past the last one the last one's); looked at only when its turn comes.
  auto key_at = [&](int b) { return sp.block(b) * KB + (lane & (KB - 1)); };
  auto seen = [&](int s) {
    return s < n_keys && (a.window == 0 || s > bmin - a.window || s < sink_keys);
  };
  auto page_at = [&](int b) { return table[min(key_at(b), n_keys - 1) >> shift]; };
  auto in_cache = [&](int page) { return (uint32_t)page < (uint32_t)a.kv.n_pages; };
  // tile b to buffer `buf`; keys that are not in the cache read page 0 (they are masked).
  // A lane computes the addresses of key (lane mod KB), and the loads take them from there.
  auto fetch = [&](int b, int page, int buf) {
    constexpr int AT_ONCE = ATT_THREADS / L::PIECES, PER_WAVE = 64 / L::PIECES;
    const uint32_t pg = in_cache(page) ? page : 0, slot = key_at(b) & page_mask;
    const uint64_t k_from = (uint64_t)kbase + pg * (uint64_t)(a.kv.k_page * 2) + slot * k_slot;
    const uint64_t v_from = (uint64_t)vbase + pg * (uint64_t)(a.kv.v_page * 2) + slot * v_slot;
#pragma unroll
    for (int i = 0; i < L::LOADS; ++i) {
      const uint32_t to = uni_int(lds0 + buf * (2 * L::BYTES) + (i * ATT_THREADS + wave * 64) * 16);
      const int key = i * AT_ONCE + tid / L::PIECES;
      const uint32_t piece = ((tid % L::PIECES) ^ L::swizzle(key)) * 16;
      if constexpr (WIDE) {
        const int first = uni_int(i * AT_ONCE + wave * PER_WAVE);
        const uint32_t mine = lane / L::PIECES;
        load_to_lds((const char*)lane_of(k_from, first), mine * k_slot + piece, to);
        load_to_lds((const char*)lane_of(v_from, first), mine * v_slot + piece, to + L::BYTES);
      } else {
        load_to_lds((const char*)shuffled(k_from, key) + piece, to);
        load_to_lds((const char*)shuffled(v_from, key) + piece, to + L::BYTES);
      }
    }
  };

  // The same for 4 bits: this thread's share of tile b, and its elements to buffer `buf`.
  using Raw = Tile4<D>;
  using G = Group4<D>;
  constexpr int KEY_SHARE = D / Raw::SHARE;  // elements of a key that a thread converts
  const int my_key = tid / Raw::SHARE, my_block = tid % Raw::SHARE * KEY_SHARE / 32;
  // values: token quarter of a group (of 4 tokens), piece, and for D = 256 which two of them
  const int my_quarter = D == 256 ? tid >> 5 : tid >> 4;
  const int my_piece = D == 256 ? (tid & 31) >> 1 : tid & 15, my_half = D == 256 ? tid & 1 : 0;
  // A wave's keys and values are those of one group of 16 tokens, or half of one: its place is
  // uniform, and a lane's places in it stay the same (addresses for each lane: prompts 707
  // rather than 691 us, with heads of 64, where registers then leave room for three blocks
  // per unit, 464 rather than 396).
  const int my_group = uni_int(wave * (KB / ATT_WAVES)) & ~(GROUP - 1);
  const uint32_t k_off = G::key(my_key & (GROUP - 1)) + tid % Raw::SHARE * (KEY_SHARE / 2);
  const uint32_t v_off = G::value(my_quarter * 4 & (GROUP - 1), my_piece) + my_half * 16;
  const uint32_t ks_off = G::key_scale(my_key & (GROUP - 1), my_block);
  const uint32_t vs_off = G::value_scale(my_quarter * 4 & (GROUP - 1), my_piece * (D / 16) / 32);
  auto load4 = [&](int b, int pages) {
    Raw t;
    const int at = __builtin_amdgcn_readlane(pages, my_group);  // lane j has the page of key j
    const uint32_t pg = in_cache(at) ? at : 0;
    const uint32_t slot = (sp.block(b) * KB + my_group) & page_mask;
    const char* g = (const char*)a.kv.k + pg * (uint64_t)a.kv.k_page + kh * a.kv.k_head +
                    (slot >> GROUP_SHIFT) * (uint64_t)a.kv.k_slot;
    if constexpr (Raw::WORDS == 4) {
      const u32x4 x = *(const u32x4*)(g + k_off), y = *(const u32x4*)(g + v_off);
#pragma unroll
      for (int i = 0; i < 4; ++i) t.k[i] = x[i], t.v[i] = y[i];
    } else {
      const u32x2 x = *(const u32x2*)(g + k_off), y = *(const u32x2*)(g + v_off);
      t.k[0] = x[0], t.k[1] = x[1], t.v[0] = y[0], t.v[1] = y[1];
    }
    t.k_scale = *(const uint8_t*)(g + ks_off);
    t.v_scale = *(const uint32_t*)(g + vs_off);
    return t;
  };
  auto store4 = [&](const Raw& t, int buf) {
    const uint32_t to = lds0 + buf * (2 * L::BYTES);
    auto place = [&](int key, int piece) {
      return to + key * (D * 2) + (piece ^ L::swizzle(key)) * 16;
    };
    // The places of neighbouring keys and pieces differ in few bits of the swizzle: they are
    // made from one place each time, since a register for each costs a block per unit.
    const float ks = scale_of(t.k_scale);
    const uint32_t k_to = place(my_key, tid % Raw::SHARE * Raw::WORDS);
#pragma unroll
    for (int i = 0; i < Raw::WORDS; ++i) write16(k_to ^ (i * 16), values8<T>(t.k[i], ks));
    auto scale = [&](int j) { return scale_of((t.v_scale >> (8 * j)) & 255); };
    if constexpr (D == 64) {  // two bytes of each token: half a 16-byte piece
      const uint32_t v_to = place(my_quarter * 4, my_piece >> 1) + (my_piece & 1) * 8;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t c = t.v[j >> 1];
        const float s = scale(j);
        const u32x2 y = j & 1 ? (u32x2){values2<T, 2>(c, s), values2<T, 3>(c, s)}
                              : (u32x2){values2<T, 0>(c, s), values2<T, 1>(c, s)};
        write8((v_to ^ (L::swizzle(j) * 16)) + L::BYTES + j * (D * 2), y);
      }
    } else if constexpr (D == 128) {
      const uint32_t v_to = place(my_quarter * 4, my_piece);
#pragma unroll
      for (int j = 0; j < 4; ++j)
        write16((v_to ^ (L::swizzle(j) * 16)) + L::BYTES + j * (D * 2),
                values8<T>(t.v[j], scale(j)));
    } else {  // 8 bytes of two tokens
      const uint32_t v_to = place(my_quarter * 4 + 2 * my_half, 2 * my_piece);
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const float s = scale_of((t.v_scale >> (16 * my_half + 8 * j)) & 255);
#pragma unroll
        for (int i = 0; i < 2; ++i)
          write16((v_to ^ (L::swizzle(j) * 16) ^ (i * 16)) + L::BYTES + j * (D * 2),
                  values8<T>(t.v[2 * j + i], s));
      }
    }
  };

  int page = 0, page_next = 0, page_far = 0;
  Raw raw;
  auto first_fetch = [&]() {
    if (b0 >= b1) return;
    if constexpr (FP4) {
      page = page_at(b0);
      store4(load4(b0, page), 0);
      if (b0 + 1 < b1) {
        page_next = page_at(b0 + 1);
        raw = load4(b0 + 1, page_next);
      }
      if (b0 + 2 < b1) page_far = page_at(b0 + 2);
      return;
    }
    page = page_at(b0);
    fetch(b0, page, 0);
    if (b0 + 1 < b1) page_next = page_at(b0 + 1);
  };
  // Without a window a prefix's keys do not depend on the rows: the first tile is on its
  // way before the rows' requests are looked up.  (A request with fewer own tokens than new
  // ones has rows that see less of it; the mask says so.)
  const bool early = plan.prefix && a.window == 0 && a.kv.n_pages > 0;
  if (plan.prefix) {
    if (early) {
      n_keys = a.prefix_len;
      sp.blocks = (n_keys + KB - 1) / KB;
      cut();
      first_fetch();
    }
    for (int i = tid; i <= a.n_req; i += ATT_THREADS) starts[i] = a.q_start[i];
  }

  // which rows: `tok` and `top` (index of the last key that it sees) of this lane's
  Request x;
  int r = 0, row0;  // row0: the block's first row among the request's (the step's) rows
  if (plan.prefix) {
    row0 = tile * TILE_ROWS;
    __syncthreads();  // the starts are in LDS
  } else {
    // Which tile: those of the requests that see most keys go first (in eight classes by
    // the keys that the request's last token sees), and in a request the last rows, so that
    // the launch does not end with a few long tiles.
    constexpr int CLASSES = 8;
    const int n = a.n_req, per = (n + ATT_THREADS - 1) / ATT_THREADS;
    const int r0 = min(n, tid * per), r1 = min(n, r0 + per);
    auto tiles_of = [&](int i, int* work) {
      const Request y = request_of(a, i);
      const int rows = min(y.q_len, a.max_q) * a.group;
      *work = a.window > 0 ? min(y.kv, a.window + min(a.n_sink, a.window)) : y.kv;
      return rows > plan.min_rows ? (rows + TILE_ROWS - 1) / TILE_ROWS : 0;
    };
    int most = 0;
    for (int i = r0; i < r1; ++i) {
      int work;
      if (tiles_of(i, &work) > 0) most = max(most, work);
    }
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) most = max(most, __shfl_xor(most, d));
    if (lane == 0) reduce[0][wave] = most;
    if (tid < CLASSES) class_tiles[tid] = 0;
    __syncthreads();
    most = max(max(reduce[0][0], reduce[0][1]), max(reduce[0][2], reduce[0][3]));
    const float scale = (float)CLASSES / (float)(most + 1);
    auto class_of = [&](int work) {  // 0: the most
      return CLASSES - 1 - min(CLASSES - 1, (int)((float)work * scale));
    };
    for (int i = r0; i < r1; ++i) {
      int work;
      const int t = tiles_of(i, &work);
      if (t > 0) atomicAdd(&class_tiles[class_of(work)], t);
    }
    __syncthreads();
    int cls = 0;
    while (cls < CLASSES && tile >= class_tiles[cls]) tile -= class_tiles[cls++];
    if (cls == CLASSES) return;  // past the last
    int sum = 0;
    for (int i = r0; i < r1; ++i) {
      int work;
      const int t = tiles_of(i, &work);
      if (t > 0 && class_of(work) == cls) sum += t;
    }
    int s = sum;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int y = __shfl_up(s, d);
      if (lane >= d) s += y;
    }
    if (lane == 63) reduce[1][wave] = s;
    __syncthreads();
    for (int w = 0; w < wave; ++w) s += reduce[1][w];
    int at = s - sum;
    if (tile >= at && tile < s) {
      for (int i = r0; i < r1; ++i) {
        int work;
        const int t = tiles_of(i, &work);
        if (t == 0 || class_of(work) != cls) continue;
        if (tile < at + t) {
          found_tile[0] = i;
          found_tile[1] = t - 1 - (tile - at);
          break;
        }
        at += t;
      }
    }
    __syncthreads();
    r = found_tile[0];
    row0 = found_tile[1] * TILE_ROWS;
    x = request_of(a, r);
    table = a.table + (int64_t)r * a.width;
  }

  int tok = 0, top = -1, qh = kh * a.group;
  bool on;
  {
    const int row = row0 + wave * 32 + col;
    const int i = row / a.group;
    const int g = row - i * a.group;
    if (plan.prefix) {
      on = i < a.n_tok;
      if (on) {
        int lo = 0, hi = a.n_req;
        while (hi - lo > 1) {
          const int mid = (lo + hi) >> 1;
          if (starts[mid] <= i) lo = mid;
          else hi = mid;
        }
        const Request y = request_of(a, lo);
        on = i >= y.q0 && i - y.q0 < min(y.q_len, a.max_q);
        top = on ? a.prefix_len + y.kv - y.q_len + (i - y.q0) : -1;
        tok = i;
      }
    } else {
      on = i < min(x.q_len, a.max_q);
      top = on ? x.kv - x.q_len + i : -1;
      tok = on ? x.q0 + i : x.q0;
    }
    if (on) qh += g;
  }
  const int n_held = plan.prefix ? a.prefix_len : x.kv;
  const int low = a.window > 0 ? top - a.window : -0x7fffffff - 1;
  // first and last key index of the wave's rows, and of the block's
  int wmin = on ? top : 0x7fffffff, wmax = on ? top : -0x7fffffff;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    wmin = min(wmin, __shfl_xor(wmin, d));
    wmax = max(wmax, __shfl_xor(wmax, d));
  }
  __syncthreads();  // reduce is read
  if (lane == 0) {
    reduce[0][wave] = wmin;
    reduce[1][wave] = wmax;
  }
  __syncthreads();
  bmin = min(min(reduce[0][0], reduce[0][1]), min(reduce[0][2], reduce[0][3]));
  const int bmax = max(max(reduce[1][0], reduce[1][1]), max(reduce[1][2], reduce[1][3]));
  wmin = uni_int(wmin);
  wmax = uni_int(wmax);

  // this part's tiles of keys
  if (!early) {
    n_keys = max(0, min(n_held, bmax + 1));
    sp = span_of<KB>(bmin, bmax, n_keys, a.window, a.n_sink, offset);
    if (bmax < 0 || a.kv.n_pages == 0) sp.blocks = 0;
    cut();
  }

  if (!early) first_fetch();

  x8 q[QC];
  {
    const elem* src =
        (const elem*)a.q + (int64_t)tok * a.q_token + (int64_t)qh * a.q_head + h * 8;
#pragma unroll
    for (int c = 0; c < QC; ++c) q[c] = *(const x8*)(src + c * 16);
  }
  f32x16 o[DT];
#pragma unroll
  for (int d = 0; d < DT; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[d][i] = 0.0f;
  float mu = NEG_INF, l = 0.0f;

  const int f = L::swizzle(col);
  uint32_t k_at[QC];  // key `col`, piece 2c + h
#pragma unroll
  for (int c = 0; c < QC; ++c)
    k_at[c] = lds0 + col * (D * 2) + ((2 * c + h) ^ f) * 16;
  uint32_t v_at[2][DT < 4 ? DT : 4];  // keys 4h + 8x + (lane mod 16) / 4, elements of tile dt
#pragma unroll
  for (int xx = 0; xx < 2; ++xx)
#pragma unroll
    for (int d = 0; d < (DT < 4 ? DT : 4); ++d) {
      const int e = lane & 15, key = 4 * h + 8 * xx + (e >> 2);
      const int piece = d * 4 + ((lane >> 4) & 1) * 2 + ((e & 3) >> 1);
      v_at[xx][d] = lds0 + L::BYTES + key * (D * 2) + (piece ^ L::swizzle(key)) * 16 + (e & 1) * 8;
    }

  for (int b = b0; b < b1; ++b) {
    const int buf = (b - b0) & 1;
    if constexpr (!FP4) wait_loads();
    __syncthreads();  // tile b is there; the other buffer is free
    const uint64_t found = __ballot(seen(key_at(b)) && in_cache(page));
    if constexpr (FP4) {
      if (b + 1 < b1) store4(raw, buf ^ 1);
      if (b + 2 < b1) raw = load4(b + 2, page_far);
      page = page_next;
      page_next = page_far;
      if (b + 3 < b1) page_far = page_at(b + 3);
    } else {
      if (b + 1 < b1) fetch(b + 1, page_next, buf ^ 1);
      page = page_next;
      if (b + 2 < b1) page_next = page_at(b + 2);
    }

    const int s0 = sp.block(b) * KB;
    const uint32_t shift_b = buf * (2 * L::BYTES);
    if (found != ~0ull) {
      // keys that are not there (the same ones for all waves): their values become 0, since
      // 0 * NaN would be NaN
#pragma unroll
      for (int i = 0; i < L::LOADS; ++i) {
        const int key = i * (ATT_THREADS / L::PIECES) + tid / L::PIECES;
        if (!((found >> key) & 1))
          write16(lds0 + shift_b + L::BYTES + (i * ATT_THREADS + tid) * 16, (u32x4){0, 0, 0, 0});
      }
      __syncthreads();
    }
    if (s0 > wmax || (a.window > 0 && s0 + KB - 1 <= wmin - a.window && s0 >= sink_keys)) continue;
    const bool full = found == ~0ull && s0 + KB - 1 <= wmin &&
                      (a.window == 0 || s0 > wmax - a.window || s0 + KB <= sink_keys);

    f32x16 s[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) s[t][i] = 0.0f;
    uint32_t k_of[QC];
#pragma unroll
    for (int c = 0; c < QC; ++c) k_of[c] = k_at[c] + shift_b;
    u32x4 kf[2][NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) kf[0][t] = read16(k_of[0] + t * 32 * D * 2);
#pragma unroll
    for (int c = 0; c < QC; ++c) {
      if (c + 1 < QC) {
#pragma unroll
        for (int t = 0; t < NT; ++t) kf[(c + 1) & 1][t] = read16(k_of[c + 1] + t * 32 * D * 2);
      }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int t = 0; t < NT; ++t)
        s[t] = T::mfma32(__builtin_bit_cast(x8, kf[c & 1][t]), q[c], s[t]);
    }
    // the values' first operands arrive while the weights are computed
    uint32_t v_of[2][DT < 4 ? DT : 4];
#pragma unroll
    for (int xx = 0; xx < 2; ++xx)
#pragma unroll
      for (int d = 0; d < (DT < 4 ? DT : 4); ++d) v_of[xx][d] = v_at[xx][d] + shift_b;
    auto values = [&](int g, int d) {
      const int more = g * 16 * D * 2 + (d / 4) * 256;
      const u32x2 lo = read_transposed(v_of[0][d % 4] + more);
      const u32x2 hi = read_transposed(v_of[1][d % 4] + more);
      return (u32x4){lo[0], lo[1], hi[0], hi[1]};
    };
    u32x4 vf[2][DT];
#pragma unroll
    for (int d = 0; d < DT; ++d) vf[0][d] = values(0, d);
    __builtin_amdgcn_sched_barrier(0);
    if (!full) {
      // the tile's keys that the lane's row sees, as bits: tested one by one they take less
      // than half the instructions of three comparisons each (chunks beside decoding requests
      // with a window, heads of 64 in 4 bits: 65.4 -> 59.8 us)
      auto below = [](int n) {  // bits 0 .. n - 1
        return n <= 0 ? 0ull : n >= 64 ? ~0ull : (1ull << n) - 1;
      };
      uint64_t mine = found & below(top - s0 + 1);
      if (a.window > 0) mine &= ~below(low - s0 + 1) | below(sink_keys - s0);
      mine >>= 4 * h;
      const uint32_t half[2] = {(uint32_t)mine, (uint32_t)(mine >> 32)};
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          s[t][i] = half[t] & (1u << (8 * (i / 4) + (i % 4))) ? s[t][i] : NEG_INF;
    }
    float mx = NEG_INF;
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[t][i]);
    mx = max_xor32(mx) * a.scale_log2 - BIAS<T>;
    if (__ballot(mx > mu + TAU)) {
      const float to = mx > mu + TAU ? mx : mu;
      const float g = part_scale(mu, to);
      mu = to;
      l *= g;
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[d][i] *= g;
    }
    const float base = mu == NEG_INF ? 0.0f : mu;
    // 16 keys at a time: the weights of the next are computed, and their values read,
    // beside the products of these
    x8 p[2];
    auto weights = [&](int g) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float e = exp2_fast(fmaf(s[g / 2][8 * (g & 1) + i], a.scale_log2, -base));
        l += e;
        p[g & 1][i] = (elem)e;  // the second product's operand (attend_common.hpp)
      }
    };
    weights(0);
#pragma unroll
    for (int g = 0; g < 2 * NT; ++g) {
      if (g + 1 < 2 * NT) {
#pragma unroll
        for (int d = 0; d < DT; ++d) vf[(g + 1) & 1][d] = values(g + 1, d);
      }
      __builtin_amdgcn_sched_barrier(0);
      if (g + 1 < 2 * NT) weights(g + 1);
#pragma unroll
      for (int d = 0; d < DT; ++d)
        o[d] = T::mfma32(__builtin_bit_cast(x8, vf[g & 1][d]), p[g & 1], o[d]);
    }
  }

  l = sum_xor32(l);
  if (plan.parts) {
    if (!on) return;
    const int64_t at = ((int64_t)part * a.n_tok + tok) * a.q_heads + qh;
    if (h == 0) plan.part_ml[at] = make_float2(mu, l);
    float* dst = plan.part_o + at * D + 4 * h;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *(f32x4*)(dst + d * 32 + i * 8) =
            (f32x4){o[d][4 * i], o[d][4 * i + 1], o[d][4 * i + 2], o[d][4 * i + 3]};
    return;
  }
  if (!on) return;
  const float inv = l > 0.0f ? 1.0f / l : l == 0.0f ? 0.0f : l;
  elem* dst = (elem*)a.out + (int64_t)tok * a.o_token + (int64_t)qh * a.o_head + 4 * h;
#pragma unroll
  for (int d = 0; d < DT; ++d)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const u32x2 y = {pack2<T>(o[d][4 * i] * inv, o[d][4 * i + 1] * inv),
                       pack2<T>(o[d][4 * i + 2] * inv, o[d][4 * i + 3] * inv)};
      *(u32x2*)(dst + d * 32 + i * 8) = y;
    }
  if (a.lse && h == 0) a.lse[(int64_t)tok * a.q_heads + qh] = (mu + log2f(l)) * LN2;
}

template <int D>
inline size_t tiles_lds(bool prefix, int n_req) {
  return 4 * (size_t)Tile<D>::BYTES + 256 + (prefix ? (size_t)(n_req + 1) * sizeof(int32_t) : 0);
}

}  // namespace fs
