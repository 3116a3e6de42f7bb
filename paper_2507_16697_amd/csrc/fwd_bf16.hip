// Ring-chunked attention forward, bf16: launches of the kernel in fwd_bf16_kernel.h without dropout.

#include "fwd_bf16_kernel.h"

namespace ringx {
namespace {

template <int D, int MODE>
hipError_t launch_plan(const FwdArgs& a) {
  const FwdPlan p = fwd_plan((a.Nq + 255) / 256 * a.BH, a.Nk, a.R, D, MODE == (int)FwdMode::kPartials);
  if constexpr (D == 64)
    if (p.cut.half) return launch<D, MODE, 1, 4>(a, p.rg, NoDrop{});
  if constexpr (MODE != (int)FwdMode::kPartials)
    if (p.cut.ks == 4) return launch<D, MODE, 4, 8>(a, p.rg, NoDrop{});
  if (p.cut.ks == 2) return launch<D, MODE, 2, 8>(a, p.rg, NoDrop{});
  return launch<D, MODE, 1, 8>(a, p.rg, NoDrop{});
}

template <int D>
hipError_t launch_mode(const FwdArgs& a, FwdMode mode) {
  switch (mode) {
    case FwdMode::kPartials: return launch_plan<D, (int)FwdMode::kPartials>(a);
    case FwdMode::kStep: return launch_plan<D, (int)FwdMode::kStep>(a);
    default: return launch_plan<D, (int)FwdMode::kFused>(a);
  }
}

}  // namespace

int64_t fwd_bf16_workgroups(int64_t BH, int64_t Nq, int64_t d) {
  (void)d;
  const int64_t bq = FwdCfg<128>::kBQ;
  static_assert(FwdCfg<128>::kBQ == FwdCfg<64>::kBQ, "one query tile size");
  return BH * ((Nq + bq - 1) / bq);
}

hipError_t launch_fwd_bf16(const FwdArgs& a, FwdMode mode) {
  return a.d == 128 ? launch_mode<128>(a, mode) : launch_mode<64>(a, mode);
}

}  // namespace ringx
