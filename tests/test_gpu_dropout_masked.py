"""Attention with dropout where keys are masked by a feature that makes their scores -inf, at the front of
the sequence or over whole ring chunks: they add nothing, whatever form the launch takes.

The reference is the fp64 oracle on the finite keys alone, at their place on the mask's key axis; the bounds
are those of test_gpu_dropout.py."""

import numpy as np
import pytest
import torch

from oracle import dropout_fp64 as od
from paper_2507_16697_amd import ring, ringx

from parity_util import to_host_f64
from test_gpu_dropout import SEED, bounds, case, check, f32_scale, state

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


@pytest.mark.parametrize("store,d", [("bf16", 64), ("bf16", 128), ("fp32", 64), ("fp32", 37)])
def test_masked_ring_chunks(store, d):
    """Chunks without a finite score before the first one that has some, and after it."""
    lengths, Nq, p, scale = (64, 96, 160, 64), 130, 0.2, f32_scale(d)
    lo, hi = 160, 320
    g, x = masked_case(40 + d, 2, Nq, sum(lengths), d, store, lo, hi)
    at = np.cumsum((0,) + lengths)
    kc = [g["k"][:, :, a:b].contiguous() for a, b in zip(at, at[1:])]
    vc = [g["v"][:, :, a:b].contiguous() for a, b in zip(at, at[1:])]
    # step by step: nothing yet, nothing yet, then the finite chunk, which the last one leaves as it is
    acc = torch.full((1, 2, Nq, d), 7.0, device="cuda")
    al = torch.full((1, 2, Nq), 7.0, device="cuda")
    seen = []
    for r, (k, v) in enumerate(zip(kc, vc)):
        ringx.ringx_attn_fwd_step_drop(g["q"], k, v, acc, al, r == 0, p, state(), int(at[r]), scale=scale)
        seen.append((acc.clone(), al.clone()))
    for a, l in seen[:2]:
        assert not a.any() and bool((l == -float("inf")).all())
    ro, rl, z = od.attention_drop(x["q"], x["k"], x["v"], scale, p, SEED, key0=lo)
    b, b_lse = bounds(x, ro, rl, z, scale, store, 2)
    for a, l in seen[2:]:
        assert (np.abs(to_host_f64(a) - ro) <= 1.01 * b["out"] + 1e-12).all()
        assert np.abs(to_host_f64(l) - rl).max() <= 2 * b_lse
    # the whole ring and its backward
    out, lse = ring.ring_forward(g["q"], kc, vc, scale=scale, dropout=(p, state()))
    dq, dk, dv = ring.ring_backward(g["q"], kc, vc, out, g["do"], lse, scale=scale, dropout=(p, state()))
    dq[..., 0] = 0.0
    dk, dv = torch.cat(dk, 2), torch.cat(dv, 2)
    for t in (dk, dv):
        assert not t[:, :, :lo].any() and not t[:, :, hi:].any()
    ref = dict(zip(("dq", "dk", "dv"), od.attention_drop_bwd(x["q"], x["k"], x["v"], ro, x["do"], rl,
                                                             scale, z)))
    ref["out"] = ro
    got = {"out": out, "dq": dq, "dk": dk[:, :, lo:hi], "dv": dv[:, :, lo:hi]}
    for name in ref:
        assert (np.abs(to_host_f64(got[name]) - ref[name]) <= 1.01 * b[name] + 1e-12).all(), name
    assert np.abs(to_host_f64(lse) - rl).max() <= 2 * b_lse
