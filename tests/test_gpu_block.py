"""A pre-norm transformer block's training step of the library's calls, on the GPU: norm -> packed projection ->
norm and rotation -> attention with dropout -> output projection with the residual -> norm -> MLP with GELU and
the residual, and all the way back.  Each part is held to the oracle on what the part before gave, to its own
bounds, so that the parts' layouts and types have to fit."""

import numpy as np
import pytest
import torch

from oracle import dropout_fp64 as od
from paper_2507_16697_amd import ringx

import test_gpu_layer_norm as ln
import test_gpu_linear as li
import test_gpu_norm_rope as nr
from parity_util import to_host_f64
from test_gpu_dropout import SEED, bounds, state

pytestmark = pytest.mark.gpu


def step(x, w, rng, H, Hkv, rot, freqs, pos, p, scale, dy, dtype):
    """Forward and backward; everything that passes between the calls."""
    t = {}
    t["a"], t["sa"] = ringx.ringx_layer_norm(x, w["n1"], w["c1"])
    t["qkv"], _ = ringx.ringx_linear(t["a"], w["wq"], w["bq"])
    rope = dict(pos=pos, q_weight=w["qn"], k_weight=w["kn"])
    t["q"], t["k"], t["v"] = ringx.ringx_qkv_norm_rope(t["qkv"], H, Hkv, freqs, rot, **rope)
    t["o"], t["lse"] = ringx.ringx_attn_fwd_drop(t["q"], t["k"], t["v"], p, rng, scale=scale)
    t["x1"], _ = ringx.ringx_linear(t["o"], w["wo"], w["bo"], residual=x)
    t["m"], t["sm"] = ringx.ringx_layer_norm(t["x1"], w["n2"], w["c2"])
    t["h"], t["z"] = ringx.ringx_linear(t["m"], w["w1"], w["b1"], act="gelu", need_pre=True)
    t["y"], _ = ringx.ringx_linear(t["h"], w["w2"], w["b2"], residual=t["x1"])
    g = {}
    g["h"], g["w2"], g["b2"] = ringx.ringx_linear_bwd(t["h"], w["w2"], dy, bias=w["b2"])
    g["m"], g["w1"], g["b1"] = ringx.ringx_linear_bwd(t["m"], w["w1"], g["h"], pre=t["z"], act="gelu", bias=w["b1"],
                                                      dx_dtype=torch.float32, dw_dtype=dtype)
    g["x1"], g["n2"], g["c2"] = ringx.ringx_layer_norm_bwd(t["x1"], g["m"], t["sm"], w["n2"], w["c2"], dres=dy)
    g["o"], g["wo"], g["bo"] = ringx.ringx_linear_bwd(t["o"], w["wo"], g["x1"], bias=w["bo"])
    g["q"], g["k"], g["v"] = ringx.ringx_attn_bwd_drop(t["q"], t["k"], t["v"], t["o"], g["o"], t["lse"], p, rng,
                                                       scale=scale)
    g["qkv"], g["qn"], g["kn"] = ringx.ringx_qkv_norm_rope_bwd(t["qkv"], g["q"], g["k"], g["v"], freqs, rot, **rope)
    g["a"], g["wq"], g["bq"] = ringx.ringx_linear_bwd(t["a"], w["wq"], g["qkv"], bias=w["bq"])
    g["x"], g["n1"], g["c1"] = ringx.ringx_layer_norm_bwd(x, g["a"], t["sa"], w["n1"], w["c1"], dres=g["x1"])
    return t, g


def make(store, B, N, H, Hkv, d, C, F, rot):
    g = np.random.default_rng(21)

    def randn(shape, std, kind=store):
        return li.dev(g.standard_normal(shape) * std, kind)

    cols = (H + 2 * Hkv) * d
    w = {"wq": randn((cols, C), C ** -0.5), "wo": randn((C, H * d), (H * d) ** -0.5), "w1": randn((F, C), C ** -0.5),
         "w2": randn((C, F), F ** -0.5), "bq": randn(cols, 0.1, "fp32"), "b1": randn(F, 0.1, "fp32"),
         "bo": randn(C, 0.1, "fp32"), "b2": randn(C, 0.1, "fp32"), "c1": randn(C, 0.1, "fp32"),
         "c2": randn(C, 0.1, "fp32")}
    for name, n in (("n1", C), ("n2", C), ("qn", d), ("kn", d)):
        w[name] = li.dev(g.uniform(0.5, 1.5, n), "fp32")
    freqs = torch.from_numpy(np.concatenate([100.0 ** (-np.arange(0, r, 2) / r) for r in rot])).cuda()
    pos = torch.from_numpy(g.integers(0, 64, (N, len(rot)), dtype=np.int32)).cuda()
    return randn((B, N, C), 1.0), w, freqs, pos, randn((B, N, C), 1.0)


@pytest.mark.parametrize("store,d,N", [("bf16", 64, 75), ("bf16", 64, 128), ("bf16", 128, 40), ("fp32", 48, 75)])
def test_a_block_and_back(store, d, N):
    B, H, Hkv, C, F, p, scale = 2, 4, 2, 200, 456, 0.2, 0.1
    rot = (d // 8 * 2,) * 3
    x, w, freqs, pos, dy = make(store, B, N, H, Hkv, d, C, F, rot)
    dtype = li.DT[store]
    t, g = step(x, w, state(), H, Hkv, rot, freqs, pos, p, scale, dy, dtype)
    # forward
    ln.check_forward(x, w["n1"], w["c1"], store, t["a"], t["sa"])
    li.check_forward(t["a"], w["wq"], w["bq"], "none", None, store, t["qkv"], None)
    rope = dict(qkv=t["qkv"], freqs=freqs, rot=rot, pos=pos, pos0=0, qw=w["qn"], kw=w["kn"])
    exact = nr.exact_of(rope)
    nr.check_forward(exact, H, Hkv, store, t["q"], t["k"], t["v"])
    y = {n: to_host_f64(v) for n, v in (("q", t["q"]), ("k", t["k"]), ("v", t["v"]), ("do", g["o"]))}
    ro, rl, z = od.attention_drop(y["q"], y["k"], y["v"], scale, p, SEED)
    b, b_lse = bounds(y, ro, rl, z, scale, store, Hkv)
    assert (np.abs(to_host_f64(t["o"]) - ro) <= 1.01 * b["out"] + 1e-12).all()
    assert np.abs(to_host_f64(t["lse"]) - rl).max() <= b_lse
    li.check_forward(t["o"], w["wo"], w["bo"], "none", x, store, t["x1"], None)
    ln.check_forward(t["x1"], w["n2"], w["c2"], store, t["m"], t["sm"])
    li.check_forward(t["m"], w["w1"], w["b1"], "gelu", None, store, t["h"], t["z"])
    li.check_forward(t["h"], w["w2"], w["b2"], "none", t["x1"], store, t["y"], None)
    # and back
    li.check_backward(t["h"], w["w2"], dy, None, "none", store, g["h"], g["w2"], g["b2"])
    li.check_backward(t["m"], w["w1"], g["h"], t["z"], "gelu", store, g["m"], g["w1"], g["b1"],
                      dw_unit=li.unit(store))
    ln.check_backward(t["x1"], g["m"], t["sm"], w["n2"], dy, store, g["x1"], g["n2"], g["c2"])
    li.check_backward(t["o"], w["wo"], g["x1"], None, "none", store, g["o"], g["wo"], g["bo"])
    ref = dict(zip(("q", "k", "v"), od.attention_drop_bwd(y["q"], y["k"], y["v"], ro, y["do"], rl, scale, z)))
    for name in ref:
        assert (np.abs(to_host_f64(g[name]) - ref[name]) <= 1.01 * b["d" + name] + 1e-12).all(), name
    nr.check_backward(exact, H, Hkv, store, (g["q"], g["k"], g["v"]), g["qkv"], g["qn"], g["kn"])
    li.check_backward(t["a"], w["wq"], g["qkv"], None, "none", store, g["a"], g["wq"], g["bq"])
    ln.check_backward(x, g["a"], t["sa"], w["n1"], g["x1"], store, g["x"], g["n1"], g["c1"])


def test_a_block_captured_and_replayed():
    B, N, H, Hkv, d, C, F, p, scale = 1, 96, 2, 2, 64, 128, 256, 0.1, 0.125
    rot = (d,)
    x, w, freqs, pos, dy = make("bf16", B, N, H, Hkv, d, C, F, rot)
    rng = state()
    args = (x, w, rng, H, Hkv, rot, freqs, pos, p, scale, dy, torch.bfloat16)
    step(*args)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(*args)
    for seed in range(3):
        g = torch.Generator(device="cuda").manual_seed(seed)
        x.copy_(torch.randn(x.shape, generator=g, device="cuda"))
        dy.copy_(torch.randn(x.shape, generator=g, device="cuda"))
        rng.add_(1)
        graph.replay()
        torch.cuda.synchronize()
        for got, want in zip(out, step(*args)):
            assert all(torch.equal(got[n], want[n]) for n in got), seed
