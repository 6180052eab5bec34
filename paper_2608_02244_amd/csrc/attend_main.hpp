// The one launch of an attention call: blocks of the rows kernel, of the tiles
// kernel over a shared prefix, and of the tiles kernel over own keys.  Where a call
// has both kinds they run side by side: the rows blocks, bound by the cache's bytes,
// come first and take one place of each compute unit, the tiles blocks, bound by the
// products, the other.
#pragma once
#include <hip/hip_runtime.h>

#include "attend_rows.hpp"
#include "attend_rows4.hpp"
#include "attend_tiles.hpp"

namespace fs {

struct MainPlan {
  int32_t rows_blocks, pre_blocks, own_blocks;  // in this order; 0: none
  RowsPlan rows;
  TilesPlan pre, own;
};

template <class T, int D, int RT, int KIND>
__device__ __forceinline__ void rows_block(const AttnArgs& a, const RowsPlan& p, int block,
                                           char* lds) {
  if constexpr (KIND == FP4_PAGES) attend_rows4<T, D, RT>(a, p, block, lds);
  else attend_rows<T, D, RT, KIND == WIDE_PAGES>(a, p, block, lds);
}

template <class T, int D, int RT, int KIND>
__global__ __launch_bounds__(ATT_THREADS, rows_occupancy(D, KIND == FP4_PAGES, RT)) void
attend_rows_kernel(AttnArgs a, MainPlan p) {
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  rows_block<T, D, RT, KIND>(a, p.rows, blockIdx.x, lds);
}

template <class T, int D, int KIND>
__global__ __launch_bounds__(ATT_THREADS, D == 256 ? 1 : 2) void attend_tiles_kernel(AttnArgs a,
                                                                                     MainPlan p) {
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  const int b = blockIdx.x;
  const bool pre = b < p.pre_blocks;
  attend_tiles<T, D, KIND>(a, pre ? p.pre : p.own, pre ? b : b - p.pre_blocks, lds);
}

template <class T, int D, int RT, int KIND>
__global__ __launch_bounds__(ATT_THREADS, D == 256 ? 1 : 2) void attend_both_kernel(AttnArgs a,
                                                                                    MainPlan p) {
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  int b = blockIdx.x;
  if (b < p.rows_blocks) {
    rows_block<T, D, RT, KIND>(a, p.rows, b, lds);
    return;
  }
  b -= p.rows_blocks;
  const bool pre = b < p.pre_blocks;
  attend_tiles<T, D, KIND>(a, pre ? p.pre : p.own, pre ? b : b - p.pre_blocks, lds);
}

inline hipError_t launch_with_lds(void (*kernel)(AttnArgs, MainPlan), dim3 grid, dim3 block,
                                  size_t lds, const AttnArgs& a, const MainPlan& p,
                                  hipStream_t s) {
  if (lds > 64 * 1024) {
    const hipError_t e = hipFuncSetAttribute(
        (const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return e;
  }
  kernel<<<grid, block, lds, s>>>(a, p);
  return hipGetLastError();
}

template <class T, int D, int RT, int KIND>
hipError_t launch_main_rows(const AttnArgs& a, const MainPlan& p, hipStream_t s) {
  const bool tiles = p.pre_blocks + p.own_blocks > 0;
  const dim3 grid((unsigned)(p.rows_blocks + p.pre_blocks + p.own_blocks)), block(ATT_THREADS);
  const size_t rl = rows_lds(a.n_req), tl = tiles_lds<D>(p.pre_blocks > 0, a.n_req);
  const size_t lds = tiles && rl < tl ? tl : rl;
  void (*kernel)(AttnArgs, MainPlan) =
      tiles ? attend_both_kernel<T, D, RT, KIND> : attend_rows_kernel<T, D, RT, KIND>;
  return launch_with_lds(kernel, grid, block, lds, a, p, s);
}

template <class T, int D, int KIND>
hipError_t launch_kind(const AttnArgs& a, const MainPlan& p, hipStream_t s) {
  if (p.rows_blocks > 0) {
    if constexpr (D <= 128)
      if (p.rows.row_tiles == 2) return launch_main_rows<T, D, 2, KIND>(a, p, s);
    return launch_main_rows<T, D, 1, KIND>(a, p, s);
  }
  const dim3 grid((unsigned)(p.pre_blocks + p.own_blocks)), block(ATT_THREADS);
  return launch_with_lds(attend_tiles_kernel<T, D, KIND>, grid, block,
                         tiles_lds<D>(p.pre_blocks > 0, a.n_req), a, p, s);
}

// One translation unit per element type and head size instantiates this, another the same
// for a cache of 4 bits.
template <class T, int D>
hipError_t launch_main(const AttnArgs& a, const MainPlan& p, hipStream_t s) {
  return a.kv.page_shift >= WIDE_SHIFT ? launch_kind<T, D, WIDE_PAGES>(a, p, s)
                                       : launch_kind<T, D, SMALL_PAGES>(a, p, s);
}

template <class T, int D>
hipError_t launch_main4(const AttnArgs& a, const MainPlan& p, hipStream_t s) {
  return launch_kind<T, D, FP4_PAGES>(a, p, s);
}

extern template hipError_t launch_main<Bf16, 64>(const AttnArgs&, const MainPlan&, hipStream_t);
extern template hipError_t launch_main<Bf16, 128>(const AttnArgs&, const MainPlan&, hipStream_t);
extern template hipError_t launch_main<Bf16, 256>(const AttnArgs&, const MainPlan&, hipStream_t);
extern template hipError_t launch_main<F16, 64>(const AttnArgs&, const MainPlan&, hipStream_t);
extern template hipError_t launch_main<F16, 128>(const AttnArgs&, const MainPlan&, hipStream_t);
extern template hipError_t launch_main<F16, 256>(const AttnArgs&, const MainPlan&, hipStream_t);
extern template hipError_t launch_main4<Bf16, 64>(const AttnArgs&, const MainPlan&, hipStream_t);
extern template hipError_t launch_main4<Bf16, 128>(const AttnArgs&, const MainPlan&, hipStream_t);
extern template hipError_t launch_main4<Bf16, 256>(const AttnArgs&, const MainPlan&, hipStream_t);
extern template hipError_t launch_main4<F16, 64>(const AttnArgs&, const MainPlan&, hipStream_t);
extern template hipError_t launch_main4<F16, 128>(const AttnArgs&, const MainPlan&, hipStream_t);
extern template hipError_t launch_main4<F16, 256>(const AttnArgs&, const MainPlan&, hipStream_t);

}  // namespace fs
