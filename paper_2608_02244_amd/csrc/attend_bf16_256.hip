// Attention kernels for bf16 elements and heads of 256.
#include "attend_main.hpp"

namespace fs {

template hipError_t launch_main<Bf16, 256>(const AttnArgs&, const MainPlan&, hipStream_t);

}  // namespace fs
