// Attention weight of held tokens: launches (attend_weight.hpp).
#include "attend_weight.hpp"

namespace fs {
namespace {

template <class T, int D, bool FP4>
hipError_t launch(const WeightArgs& a, int n_cu, hipStream_t s) {
  const size_t lds = (size_t)(ATT_WAVES + a.at.n_req + 1) * sizeof(int64_t);
  weight_rows_kernel<T, D, FP4><<<dim3((unsigned)(2 * n_cu)), ATT_THREADS, lds, s>>>(a);
  return hipGetLastError();
}

template <class T, bool FP4>
hipError_t launch_dim(const WeightArgs& a, int head_dim, int n_cu, hipStream_t s) {
  switch (head_dim) {
    case 64: return launch<T, 64, FP4>(a, n_cu, s);
    case 128: return launch<T, 128, FP4>(a, n_cu, s);
    default: return launch<T, 256, FP4>(a, n_cu, s);
  }
}

}  // namespace

size_t weight_workspace(const WeightArgs&, bool, int, int) { return 0; }

hipError_t launch_weight(const WeightArgs& a, bool fp4, int dtype, int head_dim, int n_cu, void*,
                         hipStream_t s) {
  if (n_cu <= 0) n_cu = 256;
  if (dtype == FSCHED_BF16)
    return fp4 ? launch_dim<Bf16, true>(a, head_dim, n_cu, s)
               : launch_dim<Bf16, false>(a, head_dim, n_cu, s);
  return fp4 ? launch_dim<F16, true>(a, head_dim, n_cu, s)
             : launch_dim<F16, false>(a, head_dim, n_cu, s);
}

}  // namespace fs
