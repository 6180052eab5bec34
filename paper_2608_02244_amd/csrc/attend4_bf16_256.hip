// Attention kernels for bf16 elements and heads of 256, cache of 4 bits.
#include "attend_main.hpp"

namespace fs {

template hipError_t launch_main4<Bf16, 256>(const AttnArgs&, const MainPlan&, hipStream_t);

}  // namespace fs
