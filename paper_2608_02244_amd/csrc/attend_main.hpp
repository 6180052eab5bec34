// The one launch of an attention call: blocks of the rows kernel, of the tiles
// kernel over a shared prefix, and of the tiles kernel over own keys.  Where a call
// has both kinds they run side by side: the rows blocks, bound by the cache's bytes,
// come first and take one place of each compute unit, the tiles blocks, bound by the
// products, the other.
#pragma once
#include <hip/hip_runtime.h>

#include "attend_rows.hpp"
#include "attend_tiles.hpp"

namespace fs {

struct MainPlan {
  int32_t rows_blocks, pre_blocks, own_blocks;  // in this order; 0: none
  RowsPlan rows;
  TilesPlan pre, own;
};

template <class T, int D, int RT, bool WIDE>
__global__ __launch_bounds__(ATT_THREADS, rows_occupancy(D)) void attend_rows_kernel(
    AttnArgs a, MainPlan p) {
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  attend_rows<T, D, RT, WIDE>(a, p.rows, blockIdx.x, lds);
}

template <class T, int D, bool WIDE>
__global__ __launch_bounds__(ATT_THREADS, D == 256 ? 1 : 2) void attend_tiles_kernel(AttnArgs a,
                                                                                     MainPlan p) {
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  const int b = blockIdx.x;
  const bool pre = b < p.pre_blocks;
  attend_tiles<T, D, WIDE>(a, pre ? p.pre : p.own, pre ? b : b - p.pre_blocks, lds);
}

template <class T, int D, int RT, bool WIDE>
__global__ __launch_bounds__(ATT_THREADS, D == 256 ? 1 : 2) void attend_both_kernel(AttnArgs a,
                                                                                    MainPlan p) {
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  int b = blockIdx.x;
  if (b < p.rows_blocks) {
    attend_rows<T, D, RT, WIDE>(a, p.rows, b, lds);
    return;
  }
  b -= p.rows_blocks;
  const bool pre = b < p.pre_blocks;
  attend_tiles<T, D, WIDE>(a, pre ? p.pre : p.own, pre ? b : b - p.pre_blocks, lds);
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

template <class T, int D, int RT>
hipError_t launch_main_rows(const AttnArgs& a, const MainPlan& p, hipStream_t s) {
  const bool tiles = p.pre_blocks + p.own_blocks > 0, wide = a.kv.page_shift >= WIDE_SHIFT;
  const dim3 grid((unsigned)(p.rows_blocks + p.pre_blocks + p.own_blocks)), block(ATT_THREADS);
  const size_t rl = rows_lds(a.n_req), tl = tiles_lds<D>(p.pre_blocks > 0, a.n_req);
  const size_t lds = tiles && rl < tl ? tl : rl;
  void (*kernel)(AttnArgs, MainPlan) =
      tiles ? (wide ? attend_both_kernel<T, D, RT, true> : attend_both_kernel<T, D, RT, false>)
            : (wide ? attend_rows_kernel<T, D, RT, true> : attend_rows_kernel<T, D, RT, false>);
  return launch_with_lds(kernel, grid, block, lds, a, p, s);
}

// One translation unit per element type and head size instantiates this.
template <class T, int D>
hipError_t launch_main(const AttnArgs& a, const MainPlan& p, hipStream_t s) {
  if (p.rows_blocks > 0) {
    if constexpr (D <= 128)
      if (p.rows.row_tiles == 2) return launch_main_rows<T, D, 2>(a, p, s);
    return launch_main_rows<T, D, 1>(a, p, s);
  }
  const dim3 grid((unsigned)(p.pre_blocks + p.own_blocks)), block(ATT_THREADS);
  const size_t lds = tiles_lds<D>(p.pre_blocks > 0, a.n_req);
  void (*kernel)(AttnArgs, MainPlan) = a.kv.page_shift >= WIDE_SHIFT
                                           ? attend_tiles_kernel<T, D, true>
                                           : attend_tiles_kernel<T, D, false>;
  return launch_with_lds(kernel, grid, block, lds, a, p, s);
}

extern template hipError_t launch_main<Bf16, 64>(const AttnArgs&, const MainPlan&, hipStream_t);
extern template hipError_t launch_main<Bf16, 128>(const AttnArgs&, const MainPlan&, hipStream_t);
extern template hipError_t launch_main<Bf16, 256>(const AttnArgs&, const MainPlan&, hipStream_t);
extern template hipError_t launch_main<F16, 64>(const AttnArgs&, const MainPlan&, hipStream_t);
extern template hipError_t launch_main<F16, 128>(const AttnArgs&, const MainPlan&, hipStream_t);
extern template hipError_t launch_main<F16, 256>(const AttnArgs&, const MainPlan&, hipStream_t);

}  // namespace fs
