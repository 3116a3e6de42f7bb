// Recompute backward in fp32: launches of the kernel in bwd_f32_kernel.h without dropout.

#include "bwd_f32_kernel.h"

namespace ringx {

hipError_t launch_bwd_dkdv_f32(const BwdArgs& a) { return launch_any(a, true, false, NoDrop{}); }
hipError_t launch_bwd_dq_f32(const BwdArgs& a) { return launch_any(a, false, true, NoDrop{}); }
hipError_t launch_bwd_f32(const BwdArgs& a) { return launch_any(a, true, true, NoDrop{}); }

}  // namespace ringx
