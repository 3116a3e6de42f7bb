"""Norm and rotation between a packed projection and the attention's operands, on the host: the
oracle's gradients against differences, and what the entry points refuse (CPU only)."""

import ctypes
import os

import numpy as np
import pytest

from oracle import norm_rope_fp64 as on
from paper_2507_16697_amd import ringx

needs_lib = pytest.mark.skipif(not os.path.exists(ringx.LIB_PATH), reason="libringx.so not built")
OK, NULLPTR, SHAPE, CHUNKS, UNSUP, ALIGN, WORKSPACE, HIP, ALIAS, SCRATCH, DROPOUT, ROPE = range(12)
BF16, FP32 = ringx.RINGX_BF16, ringx.RINGX_FP32
GB = 1 << 30
XP, QP, KP, VP, WP, FP, PP, GP, DP = (0x10_0000_0000 + i * 64 * GB for i in range(9))


def test_rotation_keeps_lengths_and_turns_by_position():
    g = np.random.default_rng(0)
    y = g.standard_normal((2, 5, 12))
    f, rot = g.uniform(0, 1, 5), (4, 6)
    pos = g.integers(-50, 50, (5, 2))
    z = on.turn(y, pos, f, rot)
    assert np.allclose((z ** 2).sum(-1), (y ** 2).sum(-1))
    assert np.array_equal(z[..., 10:], y[..., 10:])
    assert np.allclose(on.turn(z, pos, f, rot, back=True), y)
    # products of two rows depend on the difference of their positions alone
    a, b = g.standard_normal((2, 1, 12))
    p = np.array([[3, -4]])
    one = on.turn(a, p + 9, f, rot) @ on.turn(b, p, f, rot).T
    two = on.turn(a, p * 0 + 9, f, rot) @ on.turn(b, p * 0, f, rot).T
    assert np.allclose(one, two)


def test_oracle_gradients_are_differences():
    g = np.random.default_rng(1)
    H, Hkv, d, rot = 4, 2, 10, (4, 4)
    qkv = g.standard_normal((2, 6, (H + 2 * Hkv) * d))
    f, pos = g.uniform(0, 1, 4), g.integers(0, 40, (2, 6, 2))
    qw, kw = g.uniform(0.5, 1.5, d), g.uniform(0.5, 1.5, d)
    kwargs = dict(freqs=f, rot=rot, pos=pos, eps=1e-3)
    grads = [g.standard_normal((2, h, 6, d)) for h in (H, Hkv, Hkv)]
    dx, dqw, dkw = on.qkv_norm_rope_bwd(qkv, *grads, qw=qw, kw=kw, **kwargs)

    def loss(x, a, b):
        return sum(float((o * t).sum()) for o, t in
                   zip(on.qkv_norm_rope(x, H, Hkv, qw=a, kw=b, **kwargs), grads))

    h = 1e-5
    for name, at, grad in (("x", qkv, dx), ("qw", qw, dqw), ("kw", kw, dkw)):
        dirn = g.standard_normal(at.shape)
        x = {"x": qkv, "qw": qw, "kw": kw}
        hi, lo = dict(x), dict(x)
        hi[name], lo[name] = at + h * dirn, at - h * dirn
        num = (loss(hi["x"], hi["qw"], hi["kw"]) - loss(lo["x"], lo["qw"], lo["kw"])) / (2 * h)
        # truncation h^2 times a third derivative of order 100; cancellation 1e-14 / h
        assert abs(num - float((grad * dirn).sum())) <= 1e-7 * max(1.0, abs(num))


def fwd(x=XP, bs=1000 * 512, ts=512, qw=WP, kw=WP + 1024, f=FP, pos=PP, pbs=0, pos0=0, rot=(16, 24, 24),
        q=QP, k=KP, v=VP, B=2, N=1000, H=4, Hkv=2, d=64, eps=1e-6, dt=BF16):
    return ringx.lib().ringx_qkv_norm_rope(x, bs, ts, qw, kw, f, pos, pbs, pos0, len(rot),
                                           (ctypes.c_int64 * max(1, len(rot)))(*rot), q, k, v, B, N, H,
                                           Hkv, d, eps, dt, None)


def bwd(x=XP, bs=1000 * 512, ts=512, qw=WP, kw=WP + 1024, f=FP, pos=PP, pbs=0, pos0=0, rot=(16, 24, 24),
        q=QP, k=KP, v=VP, B=2, N=1000, H=4, Hkv=2, d=64, eps=1e-6, dt=BF16, dx=DP, dqw=GP,
        dkw=GP + 1024, ws=GP + GB, wsb=1 << 30):
    return ringx.lib().ringx_qkv_norm_rope_bwd(x, bs, ts, q, k, v, qw, kw, f, pos, pbs, pos0, len(rot),
                                               (ctypes.c_int64 * max(1, len(rot)))(*rot), dx, dqw, dkw,
                                               B, N, H, Hkv, d, eps, dt, ws, wsb, None)


@needs_lib
@pytest.mark.parametrize("fn", [fwd, bwd])
def test_refusals(fn):
    assert fn(x=0) == NULLPTR and fn(q=0) == NULLPTR and fn(v=0) == NULLPTR and fn(f=0) == NULLPTR
    assert fn(pos=0) == NULLPTR                                      # three axes need positions
    assert fn(B=0) == SHAPE and fn(N=0) == SHAPE and fn(Hkv=3) == SHAPE and fn(H=0) == SHAPE
    assert fn(N=1 << 40) == SHAPE
    assert fn(d=96) == UNSUP and fn(dt=9) == UNSUP and fn(d=129, dt=FP32) == UNSUP
    for rot in ((), (2, 2, 2, 2), (15, 24, 24), (-2, 24, 24), (32, 24, 24), (66,)):
        assert fn(rot=rot) == ROPE, rot
    for eps in (0.0, -1.0, float("nan"), float("inf")):
        assert fn(eps=eps) == ROPE
    assert fn(ts=-512) == ROPE and fn(bs=-8) == ROPE and fn(pbs=7) == ROPE
    assert fn(pos0=1 << 41) == ROPE and fn(pos0=-(1 << 41)) == ROPE
    assert fn(ts=516) == ALIGN and fn(bs=1000 * 512 + 4) == ALIGN     # bf16 rows in 16-byte pieces
    assert fn(x=XP + 8) == ALIGN and fn(qw=WP + 4) == ALIGN and fn(f=FP + 8) == ALIGN
    assert fn(pos=PP + 4) == ALIGN and fn(q=QP + 8) == ALIGN


@needs_lib
def test_refusals_of_overlaps_and_weights():
    assert fwd(q=XP + 1024) == ALIAS and fwd(k=QP) == ALIAS and fwd(v=WP) == ALIAS
    assert fwd(q=PP) == ALIAS and fwd(k=FP) == ALIAS
    assert bwd(dx=XP) == ALIAS and bwd(dx=QP) == ALIAS and bwd(dqw=DP) == ALIAS
    assert bwd(dkw=GP) == ALIAS and bwd(ws=DP) == ALIAS and bwd(ws=PP) == ALIAS
    need = ringx.ringx_qkv_norm_rope_bwd_workspace_bytes(2, 1000, 4, 2, 64, BF16)
    assert need > 0 and bwd(ws=0) == WORKSPACE and bwd(wsb=need - 1) == WORKSPACE
    # a weight and its gradient come together
    assert bwd(qw=0) == NULLPTR and bwd(dkw=0) == NULLPTR and bwd(dx=0) == NULLPTR


@needs_lib
def test_refusal_of_more_tokens_than_a_launch_takes():
    # 256 tokens to a workgroup of 2^24 - 1 at one dim per head; the last size that fits is refused for
    # another reason here (an output on top of the projection)
    most = ((1 << 24) - 1) * 256
    one = dict(B=1, H=1, Hkv=1, d=1, dt=FP32, rot=(0,), pos=None, f=None, qw=None, kw=None, bs=0, ts=0)
    assert fwd(N=most + 1, **one) == SHAPE
    assert fwd(N=most, q=XP, **one) == ALIAS


@needs_lib
def test_workspace_sizes():
    ask = ringx.ringx_qkv_norm_rope_bwd_workspace_bytes
    assert ask(0, 1, 1, 1, 64, BF16) == 0 and ask(1, 1, 3, 2, 64, BF16) == 0
    assert ask(1, 1, 1, 1, 96, BF16) == 0 and ask(1, 1, 1, 1, 129, FP32) == 0
    # bounded however many tokens
    assert 0 < ask(1, 1, 16, 16, 128, BF16) <= ask(8, 1 << 20, 16, 16, 128, BF16) <= 16 << 20


def test_binding_refuses_host_tensors():
    import torch
    x, f = torch.zeros(1, 4, 3 * 64), torch.zeros(32, dtype=torch.float64)
    with pytest.raises(ValueError, match="GPU"):
        ringx.ringx_qkv_norm_rope(x, 1, 1, f, (64,))
