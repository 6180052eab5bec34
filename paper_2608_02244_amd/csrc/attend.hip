// Attention of a step's new tokens over the paged cache (fsched_attend,
// fsched_attend_shared, fsched_attend4): which kernels a call runs, and the joining of parts.
//
//   rows blocks   requests with few rows (tokens times query heads per key head):
//                 bound by the bytes of the cache
//   tiles blocks  requests with many rows, and all tokens' rows over a shared prefix:
//                 bound by the products
//   join          a second launch, where results came in parts: a request's keys cut
//                 over waves or blocks, or a prefix and own keys
#include <hip/hip_runtime.h>

#include "attend_main.hpp"

namespace fs {
namespace {

constexpr int THREADS = 256;

struct JoinArgs {
  int row_limit;  // requests with at most this many rows were the rows kernel's, 0: none
  int slot_rows;  // rows of a slot of its parts
  int own_split;  // parts of the tiles kernel over own keys, 0: none (or results)
  int pre_split;  // parts over the prefix, 0: no prefix
  const float* rows_o;
  const float2* rows_ml;
  const RowsTile* tiles;
  const float* own_o;
  const float2* own_ml;
  const float* pre_o;
  const float2* pre_ml;
};

// Running join of parts of one row, 8 elements of it.
struct Joined {
  float m = NEG_INF, l = 0.0f, o[8] = {};
  __device__ __forceinline__ void add(float2 ml, f32x4 y, f32x4 z) {
    const float to = fmaxf(m, ml.x);
    const float f = part_scale(m, to), g = part_scale(ml.x, to);
    m = to;
    l = l * f + ml.y * g;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      o[i] = o[i] * f + y[i] * g;
      o[4 + i] = o[4 + i] * f + z[i] * g;
    }
  }
};

// Blocks for each request; D/8 threads hold a row (of any key head), and where there
// are fewer rows than that fills, several such groups share a row's parts.  Bound by
// latency (few parts) or by the parts' bytes: four parts of a row are read at once.
template <class T, int D>
__global__ __launch_bounds__(THREADS) void attend_join_kernel(AttnArgs a, JoinArgs j) {
  constexpr int LANES = D / 8, GROUPS = THREADS / LANES, AHEAD = 4;
  using elem = typename T::elem;
  using x8 = typename T::x8;
  __shared__ float other[GROUPS][D + 4];
  __shared__ float2 other_ml[GROUPS];
  const int r = blockIdx.x;
  const Request x = request_of(a, r);
  const int head_rows = min(x.q_len, a.max_q) * a.group;  // of one key head
  const bool few = head_rows <= j.row_limit;
  if (head_rows == 0 || (!few && j.own_split + j.pre_split == 0)) return;  // nothing, or written

  const int grp = threadIdx.x / LANES, d0 = (threadIdx.x % LANES) * 8;
  const int rows = head_rows * a.kv.kv_heads;
  const int per = (rows + gridDim.y - 1) / gridDim.y;  // rows of a block
  const int end = min(rows, per * ((int)blockIdx.y + 1));
  int at_once = 1;  // rows at once; GROUPS / at_once groups share one
  while (at_once < per && at_once < GROUPS) at_once *= 2;
  const int share = GROUPS / at_once, mine = grp / at_once, sub = grp % at_once;
  const int64_t all = (int64_t)a.n_tok * a.q_heads;
  for (int base = blockIdx.y * per; base < end; base += at_once) {
    const bool on = base + sub < end;
    const int kh = on ? (base + sub) / head_rows : 0;
    const int row = on ? base + sub - kh * head_rows : 0;
    const int tok = x.q0 + row / a.group, qh = kh * a.group + row % a.group;
    const int64_t th = (int64_t)tok * a.q_heads + qh;
    RowsTile t = {0, 0, 0, 0};
    if (few) t = j.tiles[(int64_t)kh * a.n_req + r];
    const int own = few ? t.count : j.own_split;
    // a single part was written as the result
    const int parts = j.pre_split == 0 && few && own <= 1 ? 0 : own + j.pre_split;
    Joined s;
    if (on) {
      for (int i0 = mine; i0 < parts; i0 += AHEAD * share) {
        float2 ml[AHEAD];
        f32x4 y[AHEAD], z[AHEAD];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
          const bool more = i0 + k * share < parts;
          const int i = more ? i0 + k * share : i0;
          const float2* from;
          const float* o;
          if (i >= own) {
            const int64_t at = (int64_t)(i - own) * all + th;
            from = j.pre_ml + at;
            o = j.pre_o + at * D;
          } else {
            const int64_t slot = i == 0 ? t.first : 2 * ((int64_t)t.wave + i);
            const int64_t at = few ? slot * j.slot_rows + row : (int64_t)i * all + th;
            from = (few ? j.rows_ml : j.own_ml) + at;
            o = (few ? j.rows_o : j.own_o) + at * D;
          }
          ml[k] = *from;
          y[k] = *(const f32x4*)(o + d0);
          z[k] = *(const f32x4*)(o + d0 + 4);
          if (!more) ml[k] = make_float2(NEG_INF, 0.0f);
        }
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) s.add(ml[k], y[k], z[k]);
      }
    }
    if (share > 1) {
      __syncthreads();
#pragma unroll
      for (int i = 0; i < 8; i += 4)
        *(f32x4*)&other[grp][d0 + i] = (f32x4){s.o[i], s.o[i + 1], s.o[i + 2], s.o[i + 3]};
      if (d0 == 0) other_ml[grp] = make_float2(s.m, s.l);
      __syncthreads();
      if (mine == 0)
        for (int i = 1; i < min(share, parts); ++i) {
          const float* o = &other[i * at_once + sub][d0];
          s.add(other_ml[i * at_once + sub], *(const f32x4*)o, *(const f32x4*)(o + 4));
        }
    }
    if (mine == 0 && on && parts > 0) {
      const float inv = s.l > 0.0f ? 1.0f / s.l : s.l == 0.0f ? 0.0f : s.l;
      x8 out;
#pragma unroll
      for (int i = 0; i < 8; ++i) out[i] = (elem)(s.o[i] * inv);
      *(x8*)((elem*)a.out + (int64_t)tok * a.o_token + (int64_t)qh * a.o_head + d0) = out;
      if (a.lse && d0 == 0) a.lse[th] = (s.m + log2f(s.l)) * LN2;
    }
  }
}

// Requests whose tables hold at most this many keys (twice as many where there are tiles for
// half the waves) are not cut over a cache of 4 bits: there is no join to launch then.  Cut /
// whole, us, requests of 1 to 64, 128, 256 and 512 keys, 8 key heads:
//     8 requests  10.4 /  8.4   10.3 /  9.2   10.9 / 13.7   11.7 / 20.4
//    64 requests  11.3 /  9.0   12.9 / 12.8   15.6 / 20.0   20.1 / 29.3
//   256 requests  19.7 / 15.2   24.7 / 18.2   30.0 / 27.1   38.0 / 41.8
//   512 requests  27.6 / 22.6   33.9 / 27.4   41.1 / 37.5   57.8 / 59.7
constexpr int WHOLE_KEYS = 128;

// What a call of this shape launches, and where its workspace's parts lie.
struct Shape {
  MainPlan main;
  JoinArgs join;
  bool joins;
  size_t bytes;
};

size_t round256(size_t b) { return (b + 255) & ~(size_t)255; }

Shape plan(const AttnArgs& a, bool fp4, int head_dim, int n_cu, char* ws) {
  Shape p;
  __builtin_memset((void*)&p, 0, sizeof(p));
  if (n_cu <= 0) n_cu = 256;
  size_t used = 0;
  auto take = [&](size_t bytes) {
    char* at = ws + used;
    used += round256(bytes);
    return ws ? at : nullptr;
  };
  const int64_t th = (int64_t)a.n_tok * a.q_heads;
  const int64_t rows = (int64_t)a.n_tok * a.group;            // rows of a key head
  const int64_t most = (int64_t)a.max_q * a.group;            // of one request, at most
  const bool prefix = a.prefix_len > 0;

  // The rows kernel holds 16 or 32 rows (16 where a head's registers are many).  With 32
  // against 16, us a call: 64 requests of 1 to 4 drafts and 8 heads per key head 82 / 158
  // (heads of 128), 51 / 120 (of 64); 32 heads per key head, 512 requests 184 / 362, 64
  // requests 51 / 45.
  const int held = head_dim == 256 ? 16 : 32;
  const bool with_rows = a.group <= held, with_tiles = most > held;
  RowsPlan& rp = p.main.rows;
  rp.row_tiles = a.group > 16 || (most > 16 && most <= held) ? 2 : 1;
  const int limit = with_rows ? 16 * rp.row_tiles : 0;
  if (with_rows) {
    // beside tiles blocks one rows block per compute unit, else as many as fit
    p.main.rows_blocks = with_tiles || prefix
                             ? n_cu
                             : n_cu * rows_occupancy(head_dim, fp4, rp.row_tiles);
    rp.waves = p.main.rows_blocks * ATT_WAVES;
    rp.most_parts = fp4 ? MOST_PARTS4 : MOST_PARTS;
    rp.keep_parts = prefix;
    const int64_t keys = (int64_t)a.width << a.kv.page_shift;
    rp.whole = fp4 && !prefix && !with_tiles &&
               keys <= (2 * (int64_t)a.n_req * a.kv.kv_heads < rp.waves ? 1 : 2) * WHOLE_KEYS;
    rp.slot_rows = most < limit ? (int)most : limit;
    const size_t whole = prefix ? (size_t)a.n_req * a.kv.kv_heads : 0;
    const size_t slots = (2 * (size_t)rp.waves + whole) * rp.slot_rows;
    rp.part_o = (float*)take(slots * head_dim * sizeof(float));
    rp.part_ml = (float2*)take(slots * sizeof(float2));
    rp.tiles = (RowsTile*)take((size_t)a.n_req * a.kv.kv_heads * sizeof(RowsTile));
    p.join.row_limit = limit;
    p.join.slot_rows = rp.slot_rows;
    p.join.rows_o = rp.part_o;
    p.join.rows_ml = rp.part_ml;
    p.join.tiles = rp.tiles;
  }
  // Keys are cut so that the places beside the rows blocks have work, none fewer than
  // 128 keys: parts cost their bytes twice (33 drafting requests behind 1,001 tokens: 25.4
  // us with 64 or 128, 27.0 with 256).
  const int64_t places = (with_rows ? 1 : 2) * (int64_t)n_cu;
  auto cut = [&](int64_t tiles, int64_t keys) {
    const int64_t want = (places + tiles * a.kv.kv_heads - 1) / (tiles * a.kv.kv_heads);
    const int64_t can = keys / 128 > 1 ? keys / 128 : 1;
    const int64_t s = want < can ? want : can;
    return (int)(s < 1 ? 1 : s);
  };
  if (with_tiles) {
    TilesPlan& t = p.main.own;
    // requests that are not the rows kernel's have more than `limit` rows each
    const int64_t big = rows / (limit + 1);
    const int64_t tiles = rows / TILE_ROWS + (big < a.n_req ? big : a.n_req);
    t.min_rows = limit;
    t.split = cut(tiles < 1 ? 1 : tiles, (int64_t)a.width << a.kv.page_shift);
    t.parts = prefix || t.split > 1;
    p.main.own_blocks = (int)((tiles < 1 ? 1 : tiles) * t.split * a.kv.kv_heads);
    if (t.parts) {
      t.part_o = (float*)take((size_t)t.split * th * head_dim * sizeof(float));
      t.part_ml = (float2*)take((size_t)t.split * th * sizeof(float2));
      p.join.own_split = t.split;
      p.join.own_o = t.part_o;
      p.join.own_ml = t.part_ml;
    }
  }
  if (prefix) {
    TilesPlan& t = p.main.pre;
    const int64_t tiles = (rows + TILE_ROWS - 1) / TILE_ROWS;
    t.prefix = 1;
    t.split = cut(tiles, a.prefix_len);
    t.parts = 1;
    p.main.pre_blocks = (int)(tiles * t.split * a.kv.kv_heads);
    t.part_o = (float*)take((size_t)t.split * th * head_dim * sizeof(float));
    t.part_ml = (float2*)take((size_t)t.split * th * sizeof(float2));
    p.join.pre_split = t.split;
    p.join.pre_o = t.part_o;
    p.join.pre_ml = t.part_ml;
  }
  p.joins = (with_rows && !rp.whole) || p.join.own_split || prefix;
  p.bytes = used;
  return p;
}

template <class T>
hipError_t main_launch(const AttnArgs& a, bool fp4, const MainPlan& p, int head_dim,
                       hipStream_t s) {
  switch (head_dim) {
    case 64: return fp4 ? launch_main4<T, 64>(a, p, s) : launch_main<T, 64>(a, p, s);
    case 128: return fp4 ? launch_main4<T, 128>(a, p, s) : launch_main<T, 128>(a, p, s);
    default: return fp4 ? launch_main4<T, 256>(a, p, s) : launch_main<T, 256>(a, p, s);
  }
}

template <class T>
void join(const AttnArgs& a, const JoinArgs& j, int head_dim, dim3 grid, hipStream_t s) {
  switch (head_dim) {
    case 64: attend_join_kernel<T, 64><<<grid, THREADS, 0, s>>>(a, j); break;
    case 128: attend_join_kernel<T, 128><<<grid, THREADS, 0, s>>>(a, j); break;
    default: attend_join_kernel<T, 256><<<grid, THREADS, 0, s>>>(a, j); break;
  }
}

}  // namespace

size_t attend_workspace(const AttnArgs& a, bool fp4, int head_dim, int n_cu) {
  return plan(a, fp4, head_dim, n_cu, nullptr).bytes;
}

hipError_t launch_attend(const AttnArgs& a, bool fp4, int dtype, int head_dim, int n_cu,
                         void* workspace, hipStream_t s) {
  const Shape p = plan(a, fp4, head_dim, n_cu, (char*)workspace);
  const hipError_t e = dtype == FSCHED_BF16 ? main_launch<Bf16>(a, fp4, p.main, head_dim, s)
                                            : main_launch<F16>(a, fp4, p.main, head_dim, s);
  if (e != hipSuccess || !p.joins) return e;
  // Enough blocks to fill the device, of 4 to 64 rows each.  Least rows of 1 / 4 / 16, us a
  // call: one request of 16,384 tokens 23 / 27 / 48, 33 drafting requests 25.8 / 25.7 /
  // 23.8, 128 requests behind a prefix 53.6 / 51.7 / 51.6.  Most rows of 16 / 64 / 256: 128
  // prompts behind a prefix 2.01 / 2.00 / 2.01 ms.
  const int64_t most = p.join.own_split + p.join.pre_split > 0 ? (int64_t)a.max_q * a.q_heads
                                                               : p.join.slot_rows * a.kv.kv_heads;
  int64_t y = (8 * n_cu + a.n_req - 1) / a.n_req;
  // A few rows of many parts each (requests of long contexts, in 4 bits) have a block each:
  // two requests of 95,000 tokens, 40 rows each, 8.6 us rather than 12.9.
  const int least = fp4 && a.n_req * most <= 2 * n_cu ? 1 : 4;
  if (y > most / least) y = most / least;
  if (y < most / 64) y = most / 64;
  if (y > 1024) y = 1024;
  if (y < 1) y = 1;
  const dim3 grid((unsigned)a.n_req, (unsigned)y);
  if (dtype == FSCHED_BF16) join<Bf16>(a, p.join, head_dim, grid, s);
  else join<F16>(a, p.join, head_dim, grid, s);
  return hipGetLastError();
}

}  // namespace fs
