// Recompute backward with dropout, bf16: dK/dV (the kernel in bwd_bf16_two_waves.h) and dQ (the one in
// bwd_dq_bf16_two_waves.h) in one launch.  Neither needs the other, and a workgroup of either fills a CU, so
// that one launch has one ragged last round where two have two, and small problems run side by side: the
// whole backward (us) in two launches -> one: 2 heads of 128, 200 x 700 32 -> 21; 8 of 64, 2048 x 2048 62 ->
// 48; 2 x 16/4 of 64, 1500 x 5003 313 -> 257; 16 of 64, 4096 x 4096 323 -> 294; 16 of 128, 4096 x 32768 even.
// dK/dV workgroups of 128 keys: at d = 64 8 waves x 64 queries (two waves per SIMD, each with the registers
// for the mask's constants; 32 queries a wave in two workgroups to a CU spill).  dQ workgroups of 8 waves x 32
// queries in KS key streams.

#define RINGX_DROPOUT
#include "bwd_bf16_two_waves.h"
#include "bwd_dq_bf16_two_waves.h"

namespace ringx {
namespace {

template <int D, int KS>
struct Forms {
  static constexpr int kQB = D == 64 ? 2 : 1;                  // 32-query blocks of a dK/dV wave
  static constexpr int kBK = D == 128 && KS == 4 ? 32 : 64;    // keys of a dQ tile
  using Dkv = dkdv::DkvCfg<D, 8, kQB>;
  using Dq = dq::DqCfg<D, KS, 8, kBK>;
  static constexpr int kDkvLds = dkdv::kLdsBytes<D, 8, kQB>, kDqLds = 4 * KS * Dq::kTileBytes;
  static constexpr int kLds = kDkvLds > kDqLds ? kDkvLds : kDqLds;
  static_assert(Dkv::kBK == 128 && Dq::kBQ == 256 / KS, "tiles of drop_bwd_workgroups");
};

// The first n_kv workgroups are dK/dV's, the others dQ's.
template <int D, int KS>
__global__ __launch_bounds__(512, 1) void bwd_drop_kernel(
    const __bf16* __restrict__ q, const __bf16* __restrict__ k, const __bf16* __restrict__ v,
    const __bf16* __restrict__ dout, const float* __restrict__ lse, const float* __restrict__ nl,
    const float* __restrict__ delta, float* __restrict__ grad_q, float* __restrict__ grad_k,
    float* __restrict__ grad_v, int BH, int H, int grp, int64_t Nq, int64_t Nk, int tiles, int n_kv, float c2,
    float scale, int accumulate_dkv, int accumulate_dq, Drop drop_kv, Drop drop_q) {
  using C = Forms<D, KS>;
  __shared__ __attribute__((aligned(1024))) char lds[C::kLds];
  if ((int)blockIdx.x < n_kv)
    dkdv::body<D, 8, C::kQB>(lds, blockIdx.x, n_kv, q, k, v, dout, nl, delta, grad_k, grad_v, BH / grp, H, grp,
                             Nq, Nk, 1, tiles, c2, scale, accumulate_dkv, drop_kv);
  else
    dq::body<D, KS, 8, C::kBK>(lds, blockIdx.x - n_kv, gridDim.x - n_kv, q, k, v, dout, lse, delta, grad_q, BH,
                              H, grp, Nq, Nk, 1, c2, scale, accumulate_dq, drop_q);
}

template <int D, int KS>
hipError_t launch(const BwdArgs& a, const Drop& drop_kv, const Drop& drop_q) {
  using C = Forms<D, KS>;
  const int64_t tiles = (a.Nk + C::Dkv::kBK - 1) / C::Dkv::kBK;
  const int64_t n_kv = a.BH / a.G * tiles * drop_kv.splits;
  const int64_t n_q = (a.Nq + C::Dq::kBQ - 1) / C::Dq::kBQ * a.BH * drop_q.splits;
  hipLaunchKernelGGL((bwd_drop_kernel<D, KS>), dim3((uint32_t)(n_kv + n_q)), dim3(512), 0, a.stream,
                     (const __bf16*)a.q, (const __bf16*)a.k, (const __bf16*)a.v, (const __bf16*)a.dout, a.lse,
                     a.nl, a.delta, a.dq, a.dk, a.dv, (int)a.BH, (int)a.H, (int)a.G, a.Nq, a.Nk, (int)tiles,
                     (int)n_kv, a.scale * kLog2e, a.scale, a.accumulate_dkv ? 1 : 0, a.accumulate_dq ? 1 : 0,
                     drop_kv, drop_q);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_bwd_drop_bf16(const BwdArgs& a, const Drop& drop_kv, const Drop& drop_q, int ks) {
  if (a.d == 128) {
    if (ks == 4) return launch<128, 4>(a, drop_kv, drop_q);
    if (ks == 2) return launch<128, 2>(a, drop_kv, drop_q);
    return launch<128, 1>(a, drop_kv, drop_q);
  }
  if (ks == 4) return launch<64, 4>(a, drop_kv, drop_q);
  if (ks == 2) return launch<64, 2>(a, drop_kv, drop_q);
  return launch<64, 1>(a, drop_kv, drop_q);
}

}  // namespace ringx
