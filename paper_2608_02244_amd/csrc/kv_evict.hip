// Pages given up by their attention weight (fsched_kv_evict).
//
// A request's pages are scored (the sum of their tokens' weights, in 64 bits, so that equal
// calls and other ways of summing agree on the choice), the n-th least score is found digit
// by digit, its row of the table closed up and its weights moved behind their pages: one
// block for each request, scores and places in LDS.  Rows of many tokens where requests are
// few are scored and moved by blocks of their own, before and behind that.  A last launch
// puts the freed pages in one list.
// Bound by latency: of a chain of some thirty barriers, of LDS and of two trips to memory.
// 8 requests of up to 2,400 tokens take 12 us (the first launch 6.6); 512 of up to 12,200 14
// (12.4; 27 with one page of a thread at a time), of which their 29 MB, at a copy's rate,
// are 6.
#include <hip/hip_runtime.h>

#include "step_common.hpp"

namespace fs {
namespace {

constexpr int THREADS = 256;
// Pages of a row that one block holds (48 KB of LDS), and tokens that it scores and moves
// rather than blocks of their own.  One block for each request beside the three launches, us,
// pages of 16: rows of 16,384 tokens 12.2 : 14.7 (1 request), 14.9 : 18.4 (16), 19.0 : 24.3
// (64); of 32,768 17.8 : 18.0, 21.9 : 23.8, 30.3 : 33.8; of 65,536 30.3 : 27.1, 35.9 : 34.0,
// 55.8 : 57.4.
constexpr int LDS_PAGES = 4096, ALONE_TOKENS = 32768;

struct Scratch {
  uint64_t* key;   // [n_req][width] scores in an order of whole numbers (not ALONE)
  int32_t* from;   // [n_req][width] old place of each page that stays (not ALONE)
  int32_t* gone;   // [n_req][width] ids of the pages given up
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

// A score as a whole number in the order of the numbers.
__device__ __forceinline__ uint64_t key_of(double sum) {
  const uint64_t b = __builtin_bit_cast(uint64_t, sum == 0.0 ? 0.0 : sum);
  return b >> 63 ? ~b : b | 1ull << 63;
}

// Lanes of a page: four tokens each in pages of 4 to 64.
__device__ __forceinline__ int lanes_of(const EvictArgs& a) {
  return 1 << min(max(a.page_shift - 2, 0), 4);
}

// Scores of a request's pages by blocks `block` of `blocks`, of N threads: four pages of each
// thread at once, since a load takes far longer than what is done with it.
template <int N, class Put>
__device__ __forceinline__ void score_pages(const EvictArgs& a, int r, const Held& h, int block,
                                            int blocks, Put put) {
  constexpr int PAGES = 4;
  const int page = 1 << a.page_shift, lanes = lanes_of(a), per = N / lanes;
  const int sub = threadIdx.x & (lanes - 1), mine = threadIdx.x / lanes;
  const float* row = a.weight + (int64_t)r * a.weight_stride + sub;
  for (int c0 = h.first + block * PAGES * per; c0 < h.last; c0 += blocks * PAGES * per) {
    double sum[PAGES] = {};
    if (page == 4 * lanes) {
      float x[PAGES][4];
#pragma unroll
      for (int p = 0; p < PAGES; ++p) {
        const int c = min(c0 + p * per + mine, h.last - 1);
#pragma unroll
        for (int i = 0; i < 4; ++i) x[p][i] = row[((int64_t)c << a.page_shift) + i * lanes];
      }
#pragma unroll
      for (int p = 0; p < PAGES; ++p)
#pragma unroll
        for (int i = 0; i < 4; ++i) sum[p] += (double)x[p][i];
    } else {
#pragma unroll
      for (int p = 0; p < PAGES; ++p) {
        const int c = min(c0 + p * per + mine, h.last - 1);
        for (int i = 0; i < page; i += lanes) sum[p] += (double)row[((int64_t)c << a.page_shift) + i];
      }
    }
    for (int d = 1; d < lanes; d <<= 1) {
#pragma unroll
      for (int p = 0; p < PAGES; ++p) sum[p] += __shfl_xor(sum[p], d);
    }
#pragma unroll
    for (int p = 0; p < PAGES; ++p) {
      const int c = c0 + p * per + mine;
      if (c < h.last && sub == 0) put(c, key_of(sum[p]));
    }
  }
}

// Weights of request r's kept tokens to places first, first + step, .. of its new row.
template <int N>
__device__ __forceinline__ void move_row(const EvictArgs& a, int r, int len, const int32_t* from,
                                         int block, int blocks) {
  const int64_t row = (int64_t)a.width << a.page_shift;
  const int page_mask = (1 << a.page_shift) - 1;
  const float* src = a.weight + (int64_t)r * a.weight_stride;
  float* dst = a.new_weight + r * row;
  auto place = [&](int64_t j) {
    return ((int64_t)from[j >> a.page_shift] << a.page_shift) | (j & page_mask);
  };
  const int64_t first = (int64_t)block * N + threadIdx.x, step = (int64_t)blocks * N;
  // read several, then write them: the compiler cannot know that the rows are apart
  constexpr int AHEAD = 4;
  if (a.page_shift >= 2 && (((uintptr_t)src | (uintptr_t)dst) & 15) == 0) {  // four at a time
    for (int64_t j0 = 4 * first; j0 < row; j0 += 4 * AHEAD * step) {
      float4 x[AHEAD];
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) {
        const int64_t j = j0 + 4 * i * step;
        x[i] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (j < len) x[i] = *(const float4*)(src + place(j));
        if (j + 1 >= len) x[i].y = 0.0f;
        if (j + 2 >= len) x[i].z = 0.0f;
        if (j + 3 >= len) x[i].w = 0.0f;
      }
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) {
        const int64_t j = j0 + 4 * i * step;
        if (j < row) *(float4*)(dst + j) = x[i];
      }
    }
  } else {
    for (int64_t j0 = first; j0 < row; j0 += AHEAD * step) {
      float x[AHEAD];
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) {
        const int64_t j = j0 + i * step;
        x[i] = j < len ? src[place(j)] : 0.0f;
      }
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) {
        const int64_t j = j0 + i * step;
        if (j < row) dst[j] = x[i];
      }
    }
  }
}

// A number that is the same in all lanes, as a scalar.
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// Sum over the block of x, and what comes before this thread.
template <int N>
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
  for (int i = 0; i < N / 64; ++i) {
    if (i < wave) s += room[i];
    total += room[i];
  }
  *before = s - x;
  return uniform(total);
}

__global__ __launch_bounds__(THREADS) void score_kernel(EvictArgs a, Scratch w) {
  const int r = blockIdx.y;
  const Held h = held_of(a, r);
  if (h.drop == 0) return;
  uint64_t* key = w.key + (int64_t)r * a.width;
  score_pages<THREADS>(a, r, h, blockIdx.x, gridDim.x, [&](int c, uint64_t k) { key[c] = k; });
}

// ALONE: scores, choice and moves of a request in this block (at most LDS_PAGES pages).
template <int N, bool ALONE>
__global__ __launch_bounds__(N) void select_kernel(EvictArgs a, Scratch w) {
  __shared__ int count[256], room[N / 64], found[3];
  __shared__ uint64_t key_room[ALONE ? LDS_PAGES : 1];
  __shared__ int32_t from_room[ALONE ? LDS_PAGES : 1];
  const int r = blockIdx.x, tid = threadIdx.x;
  const Held h = held_of(a, r);
  uint64_t* key = ALONE ? key_room : w.key + (int64_t)r * a.width;
  int32_t* from = ALONE ? from_room : w.from + (int64_t)r * a.width;
  const int32_t* table = a.table + (int64_t)r * a.width;
  if (ALONE && h.drop > 0) {
    score_pages<N>(a, r, h, 0, 1, [&](int c, uint64_t k) { key[c] = k; });
    __syncthreads();
  }
  // The drop-th least key: those below `value` go, and those equal to it up to page `until`.
  uint64_t value = 0;
  int until = 0x7fffffff;
  if (h.drop > 0) {
    int ties = h.drop, at = 56;
    for (; at >= 0; at -= 8) {
      if (tid < 256) count[tid] = 0;
      __syncthreads();
      for (int c = h.first + tid; c < h.last; c += N) {
        const uint64_t k = key[c];
        if (at == 56 || (k ^ value) >> (at + 8) == 0) atomicAdd(&count[(k >> at) & 255], 1);
      }
      __syncthreads();
      const int n = tid < 256 ? count[tid] : 0;
      int before;
      block_scan<N>(n, &before, room);
      if (before < ties && ties <= before + n) {
        found[0] = tid;
        found[1] = ties - before;
        found[2] = n;
      }
      __syncthreads();
      value |= (uint64_t)(uint32_t)uniform(found[0]) << at;
      ties = uniform(found[1]);
      if (ties == uniform(found[2])) break;  // all with these digits go
    }
    // (Set behind the loop, and from scalars: with the bits set at the break, from numbers in
    // vector registers, the compiler's code set them in every pass, by a condition bit that
    // the shift before had overwritten.)
    if (at >= 0) {
      value |= ((uint64_t)1 << at) - 1;
    } else {  // more equal ones than go: the first of them
      int equal = 0;
      for (int c0 = h.first; equal < ties; c0 += N) {
        const int c = c0 + tid;
        int before;
        const bool same = c < h.last && key[c] == value;
        const int n = block_scan<N>(same, &before, room);
        if (same && equal + before == ties - 1) found[0] = c;
        equal += n;
      }
      __syncthreads();
      until = uniform(found[0]);
    }
  }
  int32_t* to = a.new_table + (int64_t)r * a.width;
  int32_t* gone = w.gone + (int64_t)r * a.width;
  int kept = 0, freed = 0;
  for (int c0 = 0; c0 < h.pages; c0 += N) {
    const int c = c0 + tid;
    const bool on = c < h.pages;
    const bool may = h.drop > 0 && c >= h.first && c < h.last;
    const uint64_t k = may ? key[c] : 0;
    int before;
    const bool drop = may && (k < value || (k == value && c <= until));
    const int id = on ? table[c] : -1;
    // pages that stay in the low half, ids that go in the high one: at most N each
    const int both =
        block_scan<N>((int)(on && !drop) | (int)(drop && id >= 0) << 16, &before, room);
    if (on && !drop) {
      to[kept + (before & 0xffff)] = id;
      from[kept + (before & 0xffff)] = c;
    }
    if (drop && id >= 0) gone[freed + (before >> 16)] = id;
    kept += both & 0xffff;
    freed += both >> 16;
  }
  for (int c = kept + tid; c < a.width; c += N) to[c] = -1;
  const int len = h.len - (h.drop << a.page_shift);
  if (tid == 0) {
    a.new_len[r] = len;
    w.freed[r] = freed;
  }
  if (ALONE) {
    __syncthreads();
    move_row<N>(a, r, len, from, 0, 1);
  }
}

__global__ __launch_bounds__(THREADS) void move_kernel(EvictArgs a, Scratch w) {
  const int r = blockIdx.y;
  move_row<THREADS>(a, r, a.new_len[r], w.from + (int64_t)r * a.width, blockIdx.x, gridDim.x);
}

// The ids that every request gave up, one after the other.
__global__ __launch_bounds__(THREADS) void list_kernel(EvictArgs a, Scratch w) {
  __shared__ int room[THREADS / 64];
  const int r = blockIdx.x, tid = threadIdx.x;
  int sum = 0, before;
  for (int i = tid; i < r; i += THREADS) sum += w.freed[i];
  const int at = block_scan<THREADS>(sum, &before, room), n = w.freed[r];
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

// Whether one block takes each request.
bool rows_alone(const EvictArgs& a) {
  return a.width <= LDS_PAGES && (int64_t)a.width << a.page_shift <= ALONE_TOKENS;
}

Scratch scratch(const EvictArgs& a, char* ws, size_t* bytes) {
  const size_t cells = (size_t)a.n_req * a.width, shared = rows_alone(a) ? 0 : cells;
  size_t used = 0;
  auto take = [&](size_t n) {
    char* at = ws ? ws + used : nullptr;
    used += round256(n);
    return at;
  };
  Scratch w;
  w.key = (uint64_t*)take(shared * 8);
  w.from = (int32_t*)take(shared * 4);
  w.gone = (int32_t*)take(cells * 4);
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
  // no launch without the one before: it would read what that one writes
  hipError_t e;
  if (rows_alone(a)) {
    select_kernel<512, true><<<a.n_req, 512, 0, s>>>(a, w);
    e = hipGetLastError();
  } else {
    score_kernel<<<dim3(blocks(THREADS), a.n_req), THREADS, 0, s>>>(a, w);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    select_kernel<512, false><<<a.n_req, 512, 0, s>>>(a, w);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    move_kernel<<<dim3(blocks(16 * THREADS), a.n_req), THREADS, 0, s>>>(a, w);
    e = hipGetLastError();
  }
  if (e != hipSuccess) return e;
  list_kernel<<<a.n_req, THREADS, 0, s>>>(a, w);
  return hipGetLastError();
}

}  // namespace fs
