"""Attention with dropout, on the host: the oracle's generator against published vectors, its
gradients against differences, the mask's rate, and what the entry points refuse (CPU only)."""

import os

import numpy as np
import pytest

from oracle import attention_fp64 as oa
from oracle import dropout_fp64 as od
from paper_2507_16697_amd import ring, ringx

needs_lib = pytest.mark.skipif(not os.path.exists(ringx.LIB_PATH), reason="libringx.so not built")
OK, NULLPTR, SHAPE, CHUNKS, UNSUP, ALIGN, WORKSPACE, HIP, ALIAS, SCRATCH, DROPOUT, ROPE = range(12)
BF16, FP32 = ringx.RINGX_BF16, ringx.RINGX_FP32
GB = 1 << 30
QP, KP, VP, OP, LP, RP, WP = (0x10_0000_0000 + i * 64 * GB for i in range(7))   # never dereferenced


def _words(counter, key, rounds):
    return [int(x) for x in od.philox4x32([np.uint64(c) for c in counter], key, rounds)]


def test_generator_has_the_published_vectors():
    # the known-answer vectors that accompany the generator's paper
    assert _words([0] * 4, [0] * 2, 7) == [0x5f6fb709, 0x0d893f64, 0x4f121f81, 0x4f730a48]
    assert _words([0] * 4, [0] * 2, 10) == [0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8]
    ones = 0xffffffff
    assert _words([ones] * 4, [ones] * 2, 10) == [0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd]


@pytest.mark.parametrize("p", [0.0, 0.1, 0.5, 0.9])
def test_mask_rate_and_independence(p):
    rate = od.threshold(p) / 256
    m = od.keep_mask(7, 3, 5, np.arange(512), np.arange(2048), p)
    n = m.size
    sd = np.sqrt(rate * (1 - rate) / n)
    assert abs((1 - m.mean()) - rate) <= 5 * sd          # five standard deviations
    # neighbours along either axis, another head, offset or seed: products of the rates
    others = [od.keep_mask(7, 3, 6, np.arange(512), np.arange(2048), p),
              od.keep_mask(7, 4, 5, np.arange(512), np.arange(2048), p),
              od.keep_mask(8, 3, 5, np.arange(512), np.arange(2048), p)]
    pairs = [(m[:, 1:], m[:, :-1]), (m[1:], m[:-1]), (m[:, 4:], m[:, :-4]), (m[:, 32:], m[:, :-32])]
    for a, b in pairs + [(m, x) for x in others]:
        both = (~a & ~b).mean()
        assert abs(both - rate ** 2) <= 6 * np.sqrt(rate ** 2 / a.size) + 1e-12


def test_mask_is_a_function_of_place():
    whole = od.keep_mask(1, 2, 0, np.arange(100), np.arange(200), 0.3)
    part = od.keep_mask(1, 2, 0, 40 + np.arange(60), 64 + np.arange(136), 0.3)
    assert np.array_equal(part, whole[40:, 64:])


def test_oracle_without_dropout_is_plain_attention():
    g = np.random.default_rng(0)
    q, k, v = g.standard_normal((2, 3, 9, 8)), g.standard_normal((2, 3, 20, 8)), \
        g.standard_normal((2, 3, 20, 8))
    o, l, _ = od.attention_drop(q, k, v, 0.4, 0.0, (1, 2))
    ro, rl = oa.attention(q, k, v, 0.4)
    assert np.allclose(o, ro, rtol=1e-12, atol=1e-12) and np.allclose(l, rl, rtol=1e-12)


def test_oracle_gradients_are_differences():
    g = np.random.default_rng(1)
    q, k, v = g.standard_normal((1, 4, 7, 6)), g.standard_normal((1, 2, 40, 6)), \
        g.standard_normal((1, 2, 40, 6))
    do, scale, rng = g.standard_normal(q.shape), 0.3, (11, 12)
    out, lse, z = od.attention_drop(q, k, v, scale, 0.4, rng)
    grads = od.attention_drop_bwd(q, k, v, out, do, lse, scale, z)
    x = [q, k, v]
    for i in range(3):
        dirn = g.standard_normal(x[i].shape)
        h = 1e-5

        def loss(t):
            y = list(x)
            y[i] = x[i] + t * dirn
            return float((od.attention_drop(*y, scale, 0.4, rng)[0] * do).sum())

        num = (loss(h) - loss(-h)) / (2 * h)
        # truncation h^2 times a third derivative of order 10; cancellation 1e-15 / h
        assert abs(num - float((grads[i] * dirn).sum())) <= 1e-7 * max(1.0, abs(num))


def test_mask_places_of_chunks():
    assert ring.mask_places([64, 64, 32]) == [0, 64, 128]
    assert ring.mask_places([33, 1, 100]) == [0, 64, 96]


def fwd(q=QP, k=KP, v=VP, o=OP, l=LP, B=1, H=4, Hkv=2, Nq=100, Nk=300, d=64, scale=0.125, dt=BF16,
        p=0.1, rng=RP, q0=0, key0=0, ws=None, wsb=0):
    return ringx.lib().ringx_attn_fwd_drop(q, k, v, o, l, B, H, Hkv, Nq, Nk, d, scale, dt, p, rng, q0,
                                           key0, ws, wsb, None)


def fstep(q=QP, k=KP, v=VP, o=OP, l=LP, B=1, H=4, Hkv=None, Nq=100, Nk=300, d=64, scale=0.125,
          dt=BF16, p=0.1, rng=RP, q0=0, key0=0):
    return ringx.lib().ringx_attn_fwd_step_drop(q, k, v, o, l, B, H, Nq, Nk, d, scale, dt, 1, p, rng,
                                                q0, key0, None)


def bwd(q=QP, k=KP, v=VP, o=QP + 8 * GB, l=LP, B=1, H=4, Hkv=2, Nq=100, Nk=300, d=64, scale=0.125,
        dt=BF16, p=0.1, rng=RP, q0=0, key0=0, dq=OP, dk=OP + 8 * GB, dv=OP + 16 * GB,
        ws=VP + 32 * GB, wsb=1 << 20):
    return ringx.lib().ringx_attn_bwd_drop(q, k, v, o, QP + 16 * GB, l, dq, dk, dv, B, H, Hkv, Nq, Nk,
                                           d, scale, dt, p, rng, q0, key0, 0, ws, wsb, None)


def bstep(q=QP, k=KP, v=VP, o=None, l=LP, B=1, H=4, Hkv=None, Nq=100, Nk=300, d=64, scale=0.125,
          dt=BF16, p=0.1, rng=RP, q0=0, key0=0, dq=OP, dk=OP + 8 * GB, dv=OP + 16 * GB,
          delta=LP + 8 * GB):
    return ringx.lib().ringx_attn_bwd_step_drop(q, k, v, QP + 16 * GB, l, delta, dq, dk, dv, B, H, Nq,
                                                Nk, d, scale, dt, 0, 0, p, rng, q0, key0, None)


@needs_lib
@pytest.mark.parametrize("fn", [fwd, fstep, bwd, bstep])
def test_refusals(fn):
    assert fn(q=0) == NULLPTR and fn(l=0) == NULLPTR and fn(rng=0) == NULLPTR
    assert fn(B=0) == SHAPE and fn(Nq=0) == SHAPE and fn(Nk=0) == SHAPE and fn(scale=0.0) == SHAPE
    assert fn(d=96) == UNSUP and fn(dt=5) == UNSUP and fn(d=129, dt=FP32) == UNSUP
    for p in (-0.1, 1.0, 1.5, float("nan"), float("inf"), 1e-4, 0.9985):
        assert fn(p=p) == DROPOUT, p
    assert fn(q0=-1) == DROPOUT and fn(q0=(1 << 32) - 99) == DROPOUT
    assert fn(key0=-32) == DROPOUT and fn(key0=16) == DROPOUT and fn(key0=1 << 36) == DROPOUT
    assert fn(rng=RP + 4) == ALIGN and fn(q=QP + 8) == ALIGN


@needs_lib
def test_refusals_of_overlaps_and_groups():
    assert fwd(o=QP) == ALIAS and fwd(l=OP) == ALIAS and fwd(o=RP) == ALIAS and fwd(l=RP) == ALIAS
    assert fstep(o=KP) == ALIAS and fstep(l=RP) == ALIAS
    assert fwd(Hkv=3) == SHAPE and bwd(Hkv=0) == SHAPE
    need = ringx.ringx_bwd_drop_workspace_bytes(1, 4, 2, 100, 300, 64, BF16)
    assert bwd(ws=0) == WORKSPACE and bwd(wsb=need - 1) == WORKSPACE
    assert bwd(dq=QP) == ALIAS and bwd(dk=OP) == ALIAS and bwd(ws=RP) == ALIAS and bwd(dv=RP) == ALIAS
    assert bstep(dq=RP) == ALIAS and bstep(dk=OP) == ALIAS and bstep(dv=0) == NULLPTR
    pre = ringx.lib().ringx_bwd_preprocess_drop
    assert pre(QP, KP, LP, LP, 1, 2, 100, 64, BF16, 0.1, None) == ALIAS
    assert pre(QP, KP, LP, OP, 1, 2, 100, 64, BF16, 1.0, None) == DROPOUT
    assert pre(QP, 0, LP, OP, 1, 2, 100, 64, BF16, 0.1, None) == NULLPTR


@needs_lib
def test_backward_workspace_holds_the_parts():
    size, stats = ringx.ringx_bwd_drop_workspace_bytes, ringx.ringx_bwd_workspace_bytes
    # enough workgroups: the statistics alone; fp32 never splits
    for B, H, Hkv, Nq, Nk, d in ((1, 16, 16, 4096, 4096, 64), (1, 16, 16, 4096, 32768, 128),
                                 (1, 1, 1, 1, 1, 64)):
        assert size(B, H, Hkv, Nq, Nk, d, BF16) == stats(B, H, Nq, Nk, d, 1, BF16)
    assert size(1, 2, 2, 4096, 4096, 128, FP32) == stats(1, 2, 4096, 4096, 128, 1, FP32)
    # 2 heads, 4096 x 4096: two parts of dK and dV
    assert (size(1, 2, 2, 4096, 4096, 128, BF16) - stats(1, 2, 4096, 4096, 128, 1, BF16)
            == 2 * 2 * 2 * 4096 * 128 * 4)
    # the forward's: the parts' outputs and log-sum-exps, here two of 2 heads of 4096 rows
    need = ringx.ringx_fwd_drop_workspace_bytes
    assert need(1, 2, 2, 4096, 4096, 128, BF16) == 2 * 2 * 4096 * 129 * 4
    assert need(1, 2, 2, 4096, 4096, 128, FP32) == need(1, 16, 16, 4096, 4096, 64, BF16) == 0
    big = dict(H=2, Hkv=2, Nq=4096, Nk=4096, d=128)
    n = need(1, 2, 2, 4096, 4096, 128, BF16)
    assert fwd(**big) == WORKSPACE and fwd(ws=WP, wsb=n - 1, **big) == WORKSPACE
    assert fwd(ws=WP + 8, wsb=n, **big) == ALIGN
    assert fwd(ws=QP, wsb=n, **big) == ALIAS and fwd(ws=OP, wsb=n, **big) == ALIAS
    # never more parts than 512 keys and 256 query rows each allow, however few the heads
    for n in (1, 100, 255, 256, 511, 4096, 100000):
        extra = size(1, 1, 1, n, n, 64, BF16) - stats(1, 1, n, n, 64, 1, BF16)
        assert 0 <= extra <= 3 * min(32, n // 256) * n * 64 * 4
    assert size(1, 4, 3, 100, 300, 64, BF16) == 0 and size(1, 4, 2, 0, 300, 64, BF16) == 0


@needs_lib
def test_new_status_strings():
    for code in (DROPOUT, ROPE):
        assert "unknown" not in ringx.ringx_status_str(code) and code in ringx.STATUS_NAMES


def test_binding_refuses_a_wrong_generator_state():
    import torch
    t = torch.zeros(2, dtype=torch.int64)
    with pytest.raises(ValueError, match="GPU"):
        ringx._rng(t, t)


def test_calls_run_on_the_tensors_device(monkeypatch):
    """An entry point is called with its tensors' device current and that device's current stream."""
    import contextlib
    import types
    seen, current = [], [0]

    @contextlib.contextmanager
    def device(d):
        old, current[0] = current[0], d.index
        yield
        current[0] = old

    cuda = types.SimpleNamespace(current_device=lambda: current[0], device=device)
    monkeypatch.setattr(ringx, "_T", types.SimpleNamespace(cuda=cuda))
    monkeypatch.setattr(ringx, "_raw_stream", lambda d: 100 + d)
    fake = types.SimpleNamespace(entry=lambda *a: seen.append((current[0], a)) or 0)
    monkeypatch.setattr(ringx, "lib", lambda: fake)
    for index in (0, 3):
        like = types.SimpleNamespace(device=types.SimpleNamespace(index=index))
        ringx._launch("entry", like, None, 7)
        ringx._launch("entry", like, 55, 8)
    assert seen == [(0, (7, 100)), (0, (8, 55)), (3, (7, 103)), (3, (8, 55))] and current == [0]
