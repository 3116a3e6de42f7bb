"""Attention with dropout where keys are masked by a feature that makes their scores -inf at the front
of the sequence: they add nothing, whatever form the launch takes.

The reference is the fp64 oracle on the finite keys alone, at their place on the mask's key axis; the bounds
are those of test_gpu_dropout.py."""

import pytest
import torch

from paper_2507_16697_amd import ringx

from test_gpu_dropout import SEED, case, check, f32_scale, state

pytestmark = pytest.mark.gpu


def masked_case(seed, H, Nq, Nk, d, store, lo, hi):
    """Device tensors whose keys outside [lo, hi) have scores of -inf, host tensors of the others."""
    g, x = case(seed, 1, H, H, Nq, Nk, d, store)
    for t in (g, x):
        t["q"][..., 0] = 1.0
        t["k"][..., 0] = 0.0
    g["k"][:, :, :lo, 0] = -float("inf")
    g["k"][:, :, hi:, 0] = -float("inf")
    x["k"], x["v"] = x["k"][:, :, lo:hi], x["v"][:, :, lo:hi]
    return g, x


# one key stream over fewer keys than two tiles, and in a launch of more than 128 workgroups; two streams;
# four, with whole streams masked; parts of the keys, with whole parts masked
@pytest.mark.parametrize("store,H,Nq,Nk,d,lo", [
    ("bf16", 2, 70, 100, 64, 64), ("bf16", 2, 70, 100, 128, 64),
    ("bf16", 130, 70, 300, 64, 96), ("bf16", 130, 70, 300, 128, 192),
    ("bf16", 130, 270, 515, 64, 256), ("bf16", 3, 200, 400, 64, 352), ("bf16", 3, 200, 400, 128, 352),
    ("bf16", 2, 70, 2048, 64, 1056), ("bf16", 2, 70, 2048, 128, 1056),
    ("fp32", 2, 70, 100, 64, 64), ("fp32", 3, 200, 400, 36, 352), ("fp32", 1, 1, 300, 128, 288)])
def test_masked_keys_in_front(store, H, Nq, Nk, d, lo):
    print(f"masked {store} H={H} Nq={Nq} Nk={Nk} d={d} lo={lo}", flush=True)
    g, x = masked_case(3 * Nk + d, H, Nq, Nk, d, store, lo, Nk)
    p, scale = 0.2, f32_scale(d)
    out, lse = ringx.ringx_attn_fwd_drop(g["q"], g["k"], g["v"], p, state(), scale=scale)
    assert torch.isfinite(out).all() and torch.isfinite(lse).all()
    dq, dk, dv = ringx.ringx_attn_bwd_drop(g["q"], g["k"], g["v"], out, g["do"], lse, p, state(),
                                           scale=scale)
    assert not dk[:, :, :lo].any() and not dv[:, :, :lo].any()
    dq[..., 0] = 0.0      # 0 x inf by the definition; over the finite keys, whose feature is 0, it is 0
    check(x, {"out": out, "lse": lse, "dq": dq, "dk": dk[:, :, lo:], "dv": dv[:, :, lo:]}, p, SEED, scale,
          store, key0=lo)
