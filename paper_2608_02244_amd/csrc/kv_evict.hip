// Pages given up by their attention weight (fsched_kv_evict).
//
// Three launches: the pages' scores (the sum of their tokens' weights, in 64 bits, so that
// equal calls and other ways of summing agree on the choice); a block for each request that
// finds the n-th least of them digit by digit and closes its row of the table up; the
// weights moved behind their pages and the freed pages put in one list.
#include <hip/hip_runtime.h>

#include "step_common.hpp"

namespace fs {
namespace {

constexpr int THREADS = 256;

struct Scratch {
  uint64_t* key;   // [n_req][width] scores in an order of whole numbers
  int32_t* from;   // [n_req][width] old place of each page that stays
  int32_t* gone;   // [n_req][width] ids of the pages given up
  int32_t* kept;   // [n_req]
  int32_t* freed;  // [n_req] ids in `gone`
};

// What a request holds and may give up, from device data that is checked here.
struct Held {
  int len, pages;   // tokens, pages
  int first, last;  // pages that it may give up: first .. last - 1
  int drop;         // pages that it does give up
};

__device__ __forceinline__ Held held_of(const EvictArgs& a, int r) {
  const int page = 1 << a.page_shift;
  Held h;
  h.len = min(max(0, a.kv_len[r]), a.width << a.page_shift);
  h.pages = (h.len + page - 1) >> a.page_shift;
  h.first = min((int)(((int64_t)a.n_sink + page - 1) >> a.page_shift), h.pages);
  h.last = max(max(0, h.len - a.n_recent) >> a.page_shift, h.first);  // full pages only
  const int over = max(0, h.len - max(0, a.budget[r]));
  h.drop = min((over + page - 1) >> a.page_shift, h.last - h.first);
  return h;
}

// A page's lanes: as many as it has tokens, at most 64.
__global__ __launch_bounds__(THREADS) void score_kernel(EvictArgs a, Scratch w) {
  const int r = blockIdx.y;
  const Held h = held_of(a, r);
  if (h.drop == 0) return;
  const int page = 1 << a.page_shift, lanes = min(page, 64), per = THREADS / lanes;
  const int sub = threadIdx.x & (lanes - 1);
  for (int c0 = h.first + blockIdx.x * per; c0 < h.last; c0 += gridDim.x * per) {
    const int c = c0 + threadIdx.x / lanes;
    double sum = 0.0;
    if (c < h.last) {
      const float* src = a.weight + (int64_t)r * a.weight_stride + ((int64_t)c << a.page_shift);
      for (int i = sub; i < page; i += lanes) sum += (double)src[i];
    }
    for (int d = 1; d < lanes; d <<= 1) sum += __shfl_xor(sum, d);
    if (c < h.last && sub == 0) {
      const uint64_t b = __builtin_bit_cast(uint64_t, sum == 0.0 ? 0.0 : sum);
      w.key[(int64_t)r * a.width + c] = b >> 63 ? ~b : b | 1ull << 63;
    }
  }
}

// Sum over the block of x, and what comes before this thread.
__device__ __forceinline__ int block_scan(int x, int* before, int* room) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int s = x;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int y = __shfl_up(s, d);
    if (lane >= d) s += y;
  }
  __syncthreads();
  if (lane == 63) room[wave] = s;
  __syncthreads();
  int total = 0;
#pragma unroll
  for (int i = 0; i < THREADS / 64; ++i) {
    if (i < wave) s += room[i];
    total += room[i];
  }
  *before = s - x;
  return total;
}

__global__ __launch_bounds__(THREADS) void select_kernel(EvictArgs a, Scratch w) {
  __shared__ int count[256], room[THREADS / 64], found[2];
  const int r = blockIdx.x, tid = threadIdx.x;
  const Held h = held_of(a, r);
  const uint64_t* key = w.key + (int64_t)r * a.width;
  const int32_t* table = a.table + (int64_t)r * a.width;
  // The drop-th least key: `value`, of which the first `ties` go too.
  uint64_t value = 0;
  int ties = h.drop;
  if (h.drop > 0) {
    for (int at = 56; at >= 0; at -= 8) {
      count[tid] = 0;
      __syncthreads();
      for (int c = h.first + tid; c < h.last; c += THREADS) {
        const uint64_t k = key[c];
        if (at == 56 || (k ^ value) >> (at + 8) == 0) atomicAdd(&count[(k >> at) & 255], 1);
      }
      __syncthreads();
      const int n = count[tid];
      int before;
      block_scan(n, &before, room);
      if (before < ties && ties <= before + n) {
        found[0] = tid;
        found[1] = ties - before;
      }
      __syncthreads();
      value |= (uint64_t)found[0] << at;
      ties = found[1];
    }
  }
  int32_t* to = a.new_table + (int64_t)r * a.width;
  int32_t* from = w.from + (int64_t)r * a.width;
  int32_t* gone = w.gone + (int64_t)r * a.width;
  int kept = 0, freed = 0, equal = 0;
  for (int c0 = 0; c0 < h.pages; c0 += THREADS) {
    const int c = c0 + tid;
    const bool on = c < h.pages;
    const bool may = h.drop > 0 && c >= h.first && c < h.last;
    const uint64_t k = may ? key[c] : 0;
    int before;
    const int same = block_scan(may && k == value, &before, room);
    const bool drop = may && (k < value || (k == value && equal + before < ties));
    equal += same;
    const int id = on ? table[c] : -1;
    const int stay = block_scan(on && !drop, &before, room);
    if (on && !drop) {
      to[kept + before] = id;
      from[kept + before] = c;
    }
    kept += stay;
    const int go = block_scan(drop && id >= 0, &before, room);
    if (drop && id >= 0) gone[freed + before] = id;
    freed += go;
  }
  for (int c = kept + tid; c < a.width; c += THREADS) to[c] = -1;
  if (tid == 0) {
    a.new_len[r] = h.len - (h.drop << a.page_shift);
    w.kept[r] = kept;
    w.freed[r] = freed;
  }
}

__global__ __launch_bounds__(THREADS) void move_kernel(EvictArgs a, Scratch w) {
  __shared__ int room[THREADS / 64];
  const int r = blockIdx.y, tid = threadIdx.x;
  const int page_mask = (1 << a.page_shift) - 1;
  const int len = a.new_len[r];
  const int64_t row = (int64_t)a.width << a.page_shift;
  const int32_t* from = w.from + (int64_t)r * a.width;
  const float* src = a.weight + (int64_t)r * a.weight_stride;
  float* dst = a.new_weight + r * row;
  for (int64_t j = (int64_t)blockIdx.x * THREADS + tid; j < row; j += (int64_t)gridDim.x * THREADS)
    dst[j] = j < len ? src[((int64_t)from[j >> a.page_shift] << a.page_shift) | (j & page_mask)]
                     : 0.0f;
  if (blockIdx.x > 0) return;
  int sum = 0, before;
  for (int i = tid; i < r; i += THREADS) sum += w.freed[i];
  const int at = block_scan(sum, &before, room), n = w.freed[r];
  const int32_t* gone = w.gone + (int64_t)r * a.width;
  for (int i = tid; i < n; i += THREADS)
    if (at + i < a.n_freed) a.freed[at + i] = gone[i];
  if (r + 1 == a.n_req) {
    for (int i = at + n + tid; i < a.n_freed; i += THREADS) a.freed[i] = -1;
    if (tid == 0) a.count[0] = at + n;
  }
}

__global__ __launch_bounds__(THREADS) void nothing_kernel(EvictArgs a) {
  for (int i = threadIdx.x; i < a.n_freed; i += THREADS) a.freed[i] = -1;
  if (threadIdx.x == 0) a.count[0] = 0;
}

size_t round256(size_t b) { return (b + 255) & ~(size_t)255; }

Scratch scratch(const EvictArgs& a, char* ws, size_t* bytes) {
  const size_t cells = (size_t)a.n_req * a.width;
  size_t used = 0;
  auto take = [&](size_t n) {
    char* at = ws ? ws + used : nullptr;
    used += round256(n);
    return at;
  };
  Scratch w;
  w.key = (uint64_t*)take(cells * 8);
  w.from = (int32_t*)take(cells * 4);
  w.gone = (int32_t*)take(cells * 4);
  w.kept = (int32_t*)take((size_t)a.n_req * 4);
  w.freed = (int32_t*)take((size_t)a.n_req * 4);
  *bytes = used;
  return w;
}

}  // namespace

size_t evict_workspace(const EvictArgs& a) {
  size_t bytes = 0;
  if (a.n_req > 0) scratch(a, nullptr, &bytes);
  return bytes;
}

hipError_t launch_evict(const EvictArgs& a, int n_cu, void* workspace, hipStream_t s) {
  if (n_cu <= 0) n_cu = 256;
  if (a.n_req == 0) {
    nothing_kernel<<<1, THREADS, 0, s>>>(a);
    return hipGetLastError();
  }
  size_t bytes;
  const Scratch w = scratch(a, (char*)workspace, &bytes);
  const int64_t row = (int64_t)a.width << a.page_shift;
  auto blocks = [&](int64_t per) {  // of a request
    int64_t x = (row + per - 1) / per, most = (16 * (int64_t)n_cu + a.n_req - 1) / a.n_req;
    x = x < most ? x : most;
    return (unsigned)(x < 1 ? 1 : x);
  };
  score_kernel<<<dim3(blocks(THREADS), a.n_req), THREADS, 0, s>>>(a, w);
  select_kernel<<<a.n_req, THREADS, 0, s>>>(a, w);
  move_kernel<<<dim3(blocks(4 * THREADS), a.n_req), THREADS, 0, s>>>(a, w);
  return hipGetLastError();
}

}  // namespace fs
