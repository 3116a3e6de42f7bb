// Attention forward in fp32: launches of the kernel in fwd_f32_kernel.h without dropout.

#include "fwd_f32_kernel.h"

namespace ringx {

hipError_t launch_fwd_f32(const FwdArgs& a, FwdMode mode) { return launch_any(a, mode, NoDrop{}); }

}  // namespace ringx
