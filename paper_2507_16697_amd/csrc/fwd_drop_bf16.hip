// Attention forward with dropout, bf16: launches of the kernel in fwd_bf16_kernel.h with it.

#define RINGX_DROPOUT
#include "fwd_bf16_kernel.h"

namespace ringx {
namespace {

template <int D, int MODE>
hipError_t launch_plan(const FwdArgs& a, const Drop& drop) {
  const int ks = drop_fwd_streams(a.BH, a.Nq, a.Nk, D);
  if (ks == 4) return launch<D, MODE, 4, 8>(a, 1, drop);
  if (ks == 2) return launch<D, MODE, 2, 8>(a, 1, drop);
  return launch<D, MODE, 1, 8>(a, 1, drop);
}

template <int D>
hipError_t launch_mode(const FwdArgs& a, FwdMode mode, const Drop& drop) {
  if (mode == FwdMode::kStep) return launch_plan<D, (int)FwdMode::kStep>(a, drop);
  return launch_plan<D, (int)FwdMode::kFused>(a, drop);
}

}  // namespace

hipError_t launch_fwd_drop_bf16(const FwdArgs& a, FwdMode mode, const Drop& drop) {
  return a.d == 128 ? launch_mode<128>(a, mode, drop) : launch_mode<64>(a, mode, drop);
}

}  // namespace ringx
