// Attention kernels for f16 elements and heads of 128.
#include "attend_main.hpp"

namespace fs {

template hipError_t launch_main<F16, 128>(const AttnArgs&, const MainPlan&, hipStream_t);

}  // namespace fs
