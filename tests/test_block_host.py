"""Layer norm and linear layers on the host: the oracle's gradients against differences, what the entry points
refuse, and the rules that cut a product (CPU only)."""

import os
import shutil
import subprocess

import numpy as np
import pytest

from oracle import block_fp64 as ob
from paper_2507_16697_amd import build as B
from paper_2507_16697_amd import ringx

needs_lib = pytest.mark.skipif(not os.path.exists(ringx.LIB_PATH), reason="libringx.so not built")
OK, NULLPTR, SHAPE, CHUNKS, UNSUP, ALIGN, WORKSPACE, HIP, ALIAS, SCRATCH, DROPOUT, ROPE, NORM, LINEAR = range(14)
BF16, FP32 = ringx.RINGX_BF16, ringx.RINGX_FP32
GB = 1 << 30
P = [0x10_0000_0000 + i * 64 * GB for i in range(16)]


def differences(f, at, grads, h, tol):
    """Directional differences of f(**at) for every name of grads."""
    g = np.random.default_rng(5)
    for name, grad in grads.items():
        dirn = g.standard_normal(at[name].shape)
        hi, lo = dict(at), dict(at)
        hi[name], lo[name] = at[name] + h * dirn, at[name] - h * dirn
        num = (f(**hi) - f(**lo)) / (2 * h)
        assert abs(num - float((grad * dirn).sum())) <= tol * max(1.0, abs(num)), name


def test_oracle_layer_norm_gradients_are_differences():
    g = np.random.default_rng(1)
    x, w, b = g.standard_normal((3, 4, 7)), g.uniform(0.5, 1.5, 7), g.standard_normal(7)
    dy, dres = g.standard_normal((2, 3, 4, 7))
    y, mean, r = ob.layer_norm(x, w, b, 1e-2)
    assert np.allclose(((y - b) / w).mean(-1), 0, atol=1e-12)
    dx, dw, db = ob.layer_norm_bwd(x, dy, mean, r, w, dres)
    # truncation h^2 times a third derivative of order 100; cancellation 1e-14 / h
    differences(lambda x, w, b: float((ob.layer_norm(x, w, b, 1e-2)[0] * dy).sum() + (x * dres).sum()),
                {"x": x, "w": w, "b": b}, {"x": dx, "w": dw, "b": db}, 1e-5, 1e-7)


@pytest.mark.parametrize("act", list(ringx.ACTIVATIONS))
@pytest.mark.parametrize("heads", [0, 2])
def test_oracle_linear_gradients_are_differences(act, heads):
    g = np.random.default_rng(2)
    x = g.standard_normal((2, 2, 5, 3)) if heads else g.standard_normal((2, 5, 6))
    w, b, res, dy = (g.standard_normal(s) for s in ((4, 6), (4,), (2, 5, 4), (2, 5, 4)))
    y, z = ob.linear(x, w, b, act, res)
    assert np.allclose(y, ob.act(z, act) + res.reshape(10, 4))
    dx, dw, db = ob.linear_bwd(x, w, dy, z, act)
    differences(lambda x, w, b: float((ob.linear(x, w, b, act, res)[0] * dy.reshape(10, 4)).sum()),
                {"x": x, "w": w, "b": b}, {"x": dx, "w": dw, "b": db}, 1e-5, 1e-7)


def test_oracle_against_torch():
    import torch
    import torch.nn.functional as F
    g = np.random.default_rng(3)
    x, w, b = (torch.from_numpy(g.standard_normal(s)) for s in ((5, 8), (8,), (8,)))
    assert np.allclose(ob.layer_norm(x.numpy(), w.numpy(), b.numpy())[0], F.layer_norm(x, (8,), w, b).numpy())
    z = torch.linspace(-6, 6, 101, dtype=torch.float64)
    for name, f in (("gelu", F.gelu), ("gelu_tanh", lambda t: F.gelu(t, approximate="tanh")), ("silu", F.silu)):
        assert np.allclose(ob.act(z.numpy(), name), f(z).numpy(), atol=1e-14)


def norm(x=P[0], stride=512, w=P[1], b=P[2], y=P[3], stats=P[4], rows=100, C=512, eps=1e-5, dt=BF16):
    return ringx.lib().ringx_layer_norm(x, stride, w, b, y, stats, rows, C, eps, dt, None)


def norm_bwd(x=P[0], stride=512, dy=P[1], dres=P[2], w=P[3], stats=P[4], dx=P[5], dw=P[6], db=P[7], rows=100,
             C=512, dt=BF16, dyt=None, ws=P[8], wsb=GB):
    return ringx.lib().ringx_layer_norm_bwd(x, stride, dy, dres, w, stats, dx, dw, db, rows, C, dt,
                                            dt if dyt is None else dyt, ws, wsb, None)


@needs_lib
@pytest.mark.parametrize("fn", [norm, norm_bwd])
def test_norm_refusals(fn):
    assert fn(x=0) == NULLPTR
    assert fn(rows=0) == SHAPE and fn(rows=-3) == SHAPE and fn(rows=1 << 40) == SHAPE
    assert fn(dt=7) == UNSUP
    assert fn(C=0) == NORM and fn(C=16385, stride=1 << 15) == NORM and fn(stride=511) == NORM
    assert fn(stride=1 << 38) == SHAPE
    assert fn(x=P[0] + 8) == ALIGN and fn(w=P[1] + 1 * GB + 4) == ALIGN
    # a stride is not looked at for one row
    assert fn(rows=1, stride=0, x=P[0] + 8) == ALIGN


@needs_lib
def test_norm_refusals_of_each_way():
    assert norm(y=0) == NULLPTR
    for eps in (-1e-9, float("nan"), float("inf")):
        assert norm(eps=eps) == NORM
    assert norm(y=P[0] + 512) == ALIAS and norm(stats=P[3] + 1024) == ALIAS and norm(y=P[1]) == ALIAS
    # rows behind one another up to the last one's end
    assert norm(y=P[0] + 99 * 1040 + 1024 - 16, stride=520) == ALIAS
    assert norm_bwd(dy=0) == NULLPTR and norm_bwd(stats=0) == NULLPTR and norm_bwd(dx=0) == NULLPTR
    need = ringx.ringx_layer_norm_bwd_workspace_bytes(100, 512, BF16)
    assert need > 0 and norm_bwd(ws=0) == WORKSPACE and norm_bwd(wsb=need - 1) == WORKSPACE
    assert norm_bwd(dx=P[1]) == ALIAS and norm_bwd(dx=P[2]) == ALIAS and norm_bwd(dw=P[7]) == ALIAS
    assert norm_bwd(dyt=5) == UNSUP and norm_bwd(dt=FP32, dyt=BF16) == UNSUP
    # an fp32 gradient is twice as long
    assert norm_bwd(dx=P[1] + 102400, dyt=FP32) == ALIAS
    assert norm_bwd(ws=P[5]) == ALIAS and norm_bwd(db=P[4]) == ALIAS and norm_bwd(ws=P[8] + 8) == ALIGN
    ask = ringx.ringx_layer_norm_bwd_workspace_bytes
    assert ask(0, 8, BF16) == 0 and ask(8, 16385, BF16) == 0 and ask(8, 8, 5) == 0
    assert ask(1 << 30, 16384, BF16) <= 128 << 20


def lin(x=P[0], stride=512, heads=0, tokens=0, w=P[1], b=P[2], res=P[3], y=P[4], pre=P[5], M=300, K=512, O=256,
        act=1, dt=BF16, ws=P[6], wsb=GB):
    return ringx.lib().ringx_linear(x, stride, heads, tokens, w, b, res, y, pre, M, K, O, act, dt, ws, wsb, None)


def lin_bwd(x=P[0], stride=512, heads=0, tokens=0, w=P[1], dy=P[2], pre=P[3], dx=P[4], dw=P[5], db=P[6], M=300,
            K=512, O=256, act=1, dt=BF16, dxt=None, dwt=FP32, acc=0, ws=P[7], wsb=GB):
    return ringx.lib().ringx_linear_bwd(x, stride, heads, tokens, w, dy, pre, dx, dw, db, M, K, O, act, dt,
                                        dt if dxt is None else dxt, dwt, acc, ws, wsb, None)


@needs_lib
@pytest.mark.parametrize("fn", [lin, lin_bwd])
def test_linear_refusals(fn):
    assert fn(x=0) == NULLPTR and fn(w=0) == NULLPTR
    assert fn(M=0) == SHAPE and fn(dt=4) == UNSUP and fn(act=4) == LINEAR and fn(act=-1) == LINEAR
    assert fn(K=0) == LINEAR and fn(O=0) == LINEAR and fn(K=(1 << 20) + 1, stride=1 << 21) == LINEAR
    assert fn(O=(1 << 20) + 1) == LINEAR and fn(M=(1 << 31) - 1023) == LINEAR and fn(stride=511) == LINEAR
    assert fn(heads=-1) == LINEAR and fn(heads=3, tokens=100) == LINEAR and fn(heads=2, tokens=0) == LINEAR
    assert fn(heads=2, tokens=7) == LINEAR
    assert fn(stride=1 << 38) == SHAPE and fn(M=(1 << 31) - 1024, K=8192, stride=8192) == SHAPE
    assert fn(x=P[0] + 8) == ALIGN and fn(w=P[1] + 2) == ALIGN
    # more tiles than a launch takes, each product's
    assert fn(M=(1 << 31) - 1024, K=8, stride=8, O=136) == SHAPE
    assert fn(M=128, K=1 << 20, stride=1 << 20, O=1 << 20) == SHAPE


@needs_lib
def test_linear_refusals_of_each_way():
    assert lin(y=0) == NULLPTR and lin(y=P[0] + 1024) == ALIAS and lin(pre=P[4] + 16) == ALIAS
    assert lin(y=P[3]) == ALIAS and lin(y=P[2]) == ALIAS and lin(b=P[2] + 4) == ALIGN
    # operands that have to be copied need a workspace
    need = ringx.ringx_linear_workspace_bytes(511, 0, 0, 300, 511, 256, BF16)
    assert need > 0 and lin(K=511, ws=0) == WORKSPACE and lin(K=511, wsb=need - 1) == WORKSPACE
    assert lin(K=511, ws=P[1]) == ALIAS and lin(K=511, ws=P[6] + 8) == ALIGN
    assert lin_bwd(dy=0) == NULLPTR and lin_bwd(dx=0, dw=0, db=0) == NULLPTR
    # what the activation's derivative needs, and nothing where there is none
    assert lin_bwd(pre=0) == NULLPTR and lin_bwd(act=0) == NULLPTR
    assert lin_bwd(dwt=5) == UNSUP and lin_bwd(dt=FP32, dwt=BF16) == UNSUP and lin_bwd(dwt=BF16, acc=1) == UNSUP
    assert lin_bwd(dxt=5) == UNSUP and lin_bwd(dt=FP32, dxt=BF16) == UNSUP
    assert lin_bwd(dxt=FP32, heads=2, tokens=100) == UNSUP
    need = ringx.ringx_linear_bwd_workspace_bytes(512, 0, 0, 300, 512, 256, 1, BF16)
    assert need > 0 and lin_bwd(ws=0) == WORKSPACE and lin_bwd(wsb=need - 1) == WORKSPACE
    assert lin_bwd(dx=P[2]) == ALIAS and lin_bwd(dw=P[4]) == ALIAS and lin_bwd(db=P[3]) == ALIAS
    assert lin_bwd(ws=P[0]) == ALIAS and lin_bwd(dx=P[4] + 4) == ALIGN
    assert ringx.ringx_linear_workspace_bytes(8, 0, 0, 0, 8, 8, BF16) == 0
    assert ringx.ringx_linear_bwd_workspace_bytes(8, 0, 0, 8, 8, 8, 9, BF16) == 0


@needs_lib
def test_status_text():
    assert "row length" in ringx.ringx_status_str(NORM) and "activation" in ringx.ringx_status_str(LINEAR)


def test_binding_refuses_host_tensors():
    import torch
    x, w = torch.zeros(4, 8), torch.zeros(8, 8)
    for call in (lambda: ringx.ringx_layer_norm(x), lambda: ringx.ringx_linear(x, w),
                 lambda: ringx.ringx_linear(x.view(1, 2, 2, 8), torch.zeros(8, 16)),
                 lambda: ringx.ringx_linear_bwd(x, w, x), lambda: ringx.ringx_layer_norm_bwd(x, x, x)):
        with pytest.raises(ValueError, match="GPU"):
            call()


# The rules that cut a product, compiled and asked on the host.
MAIN = r"""
#include <cstdio>
#include "ringx_kernels.h"
int main() {
  using namespace ringx;
  long long kind, a, b, c;
  while (std::scanf("%lld %lld %lld %lld", &kind, &a, &b, &c) == 4) {
    GemmCut x, y;
    bool pair = false;
    if (kind == 0) {
      x = gemm_cut(a, b, c);
    } else {   // M, K, O
      x = gemm_cut(a, b, c), y = gemm_cut(c, b, a);
      pair = gemm_cut_pair(a, b, c, &x, &y);
    }
    std::printf("%d %d %u %u %lld %d %u %u %lld\n", (int)x.large, x.groups, x.whole, x.parts,
                (long long)x.part_bytes, (int)pair, y.whole, y.parts, (long long)y.part_bytes);
  }
}
"""


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    if shutil.which("g++") is None or not os.path.isdir("/opt/rocm/include"):
        pytest.skip("needs g++ and the HIP headers")
    d = tmp_path_factory.mktemp("rules")
    (d / "main.cpp").write_text(MAIN)
    r = subprocess.run(["g++", "-std=c++17", "-O1", "-D__HIP_PLATFORM_AMD__", "-I", "/opt/rocm/include", "-I",
                        B.CSRC, "-I", B.INCLUDE, str(d / "main.cpp"), "-o", str(d / "main")],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]

    def ask(rows):
        out = subprocess.run([str(d / "main")], input="\n".join(" ".join(map(str, r)) for r in rows),
                             capture_output=True, text=True, timeout=60).stdout.split("\n")
        return [tuple(map(int, line.split())) for line in out if line]
    return ask


def test_cuts_cover_every_tile_and_fit(rules):
    g = np.random.default_rng(11)
    sizes = [tuple(int(round(2 ** g.uniform(0, 15))) for _ in range(3)) for _ in range(400)]
    for (I, J, R), (large, groups, whole, parts, nbytes, *_) in zip(sizes, rules([(0, *s) for s in sizes])):
        side, slots = (256, 256) if large else (128, 512)
        tiles = -(-I // side) * -(-J // side)
        assert whole <= tiles and parts >= 1 and groups in (1, 2)
        rest = tiles - whole
        if parts == 1:
            assert rest == 0 and nbytes == 0
        else:
            # no part without a step, no more of them than are at work at a time
            assert 0 < rest * parts <= slots and parts <= -(-R // 64)
            assert nbytes == rest * parts * side * side * 4
        if groups == 2:
            assert not large and whole + rest * parts <= 256


def test_pairs_fit_one_round(rules):
    g = np.random.default_rng(12)
    sizes = [tuple(int(round(2 ** g.uniform(0, 13))) for _ in range(3)) for _ in range(400)]
    some = 0
    for (M, K, O), (large, groups, w1, p1, b1, pair, w2, p2, b2) in zip(sizes, rules([(1, *s) for s in sizes])):
        if not pair:
            continue
        some += 1
        n1, n2 = -(-M // 128) * -(-K // 128), -(-O // 128) * -(-K // 128)
        assert not large and n1 * p1 + n2 * p2 <= (256 if groups == 2 else 512)
        assert (w1, w2) == (n1 if p1 == 1 else 0, n2 if p2 == 1 else 0)
        assert p1 <= -(-O // 64) and p2 <= -(-M // 64)
        assert b1 == (n1 * p1 * 65536 if p1 > 1 else 0) and b2 == (n2 * p2 * 65536 if p2 > 1 else 0)
    assert some > 50


def test_large_products_take_large_tiles_whole(rules):
    for sizes in ((8192, 8192, 8192), (32768, 6144, 2048), (16384, 8192, 2048), (8192, 2048, 16384)):
        large, groups, whole, parts, *_ = rules([(0, *sizes)])[0]
        assert (large, groups, parts) == (1, 1, 1) and whole == sizes[0] * sizes[1] // 65536
