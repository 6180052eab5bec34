// Attention kernels for f16 elements and heads of 256.
#include "attend_main.hpp"

namespace fs {

template hipError_t launch_main<F16, 256>(const AttnArgs&, const MainPlan&, hipStream_t);

}  // namespace fs
