"""Layer norm, forward and backward, on the GPU against the fp64 oracle.

Bounds are those of rounding.  E = 2^-24 is half a step of fp32.  A thread adds at most 32 values one after
the other and a row's threads in at most 9 more steps: a sum of a row is off by at most 41 E of the sum of its
terms' sizes."""

import numpy as np
import pytest
import torch

from oracle import block_fp64 as ob
from paper_2507_16697_amd import ringx

from parity_util import to_host_f64

pytestmark = pytest.mark.gpu

E = 2.0 ** -24
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}


def unit(store):
    return 2.0 ** -8 if store == "bf16" else 0.0


def make(seed, shape, store, pad=0, mean=0.5, spread=1.0):
    g = np.random.default_rng(seed)
    C = shape[-1]
    wide = g.standard_normal((*shape[:-1], C + pad)) * spread * np.exp(g.uniform(-1, 1, C + pad)) + mean
    x = torch.from_numpy(wide.astype(np.float32)).to(DT[store]).cuda()[..., :C]
    w, b = (torch.from_numpy(g.uniform(-1.5, 1.5, C).astype(np.float32)).cuda() for _ in range(2))
    dy, dres = (torch.from_numpy(g.standard_normal(shape).astype(np.float32)).to(DT[store]).cuda()
                for _ in range(2))
    return x, w, b, dy, dres


def f64(t):
    return None if t is None else to_host_f64(t)


def check_forward(x, w, b, store, y, stats, eps=1e-5):
    X, W, B = f64(x), f64(w), f64(b)
    ref, mean, r = ob.layer_norm(X, W, B, eps)
    n = (X - mean[..., None]) * r[..., None]
    aw = 1.0 if W is None else np.abs(W)
    # the mean's 41 E of a deviation, r's 27 E (half of the squares' 45 E, its root and quotient), and the
    # differences', products' and the last sum's own roundings
    bound = E * (45 * aw + 34 * np.abs(n) * aw + 3 * np.abs(ref)) + unit(store) * np.abs(ref)
    err = np.abs(f64(y) - ref)
    assert np.isfinite(err).all() and (err <= 1.01 * bound + 1e-30).all(), float((err - bound).max())
    if stats is not None:
        s = f64(stats).reshape(2, *mean.shape)
        assert (np.abs(s[0] - mean) <= 1.01 * E * (np.abs(mean) + 45 / r)).all()
        assert (np.abs(s[1] - r) <= 1.01 * 27 * E * r).all()


def check_backward(x, dy, stats, w, dres, store, dx, dw, db):
    X, G, W = f64(x), f64(dy), f64(w)
    s = f64(stats).reshape(2, *X.shape[:-1])
    ref, rw, rb = ob.layer_norm_bwd(X, G, s[0], s[1], W, f64(dres))
    r = s[1][..., None]
    n = np.abs((X - s[0][..., None]) * r)
    g = np.abs(G if W is None else G * W)
    m1, m2 = g.mean(-1, keepdims=True), (g * n).mean(-1, keepdims=True)
    bound = E * r * (4 * g + 44 * m1 + 50 * n * m2) + E * np.abs(ref) + unit(store) * np.abs(ref)
    if dres is not None:
        bound = bound + E * np.abs(f64(dres))
    err = np.abs(f64(dx) - ref)
    assert np.isfinite(err).all() and (err <= 1.01 * bound + 1e-30).all(), float((err - bound).max())
    axes = tuple(range(X.ndim - 1))
    rows = X.size // X.shape[-1]
    for got, want, size in ((dw, rw, (np.abs(G) * n).sum(axes)), (db, rb, np.abs(G).sum(axes))):
        if got is not None:
            err = np.abs(f64(got) - want)
            assert np.isfinite(err).all() and (err <= (rows + 8) * E * size + 1e-30).all()


SHAPES = [
    # every width class of the kernels, its edges, and widths that fit no piece
    ((1, 8), 0), ((1, 2048), 0), ((7, 1), 0), ((5, 3), 4), ((9, 64), 0), ((33, 65), 0), ((37, 72), 8),
    ((130, 128), 0), ((65, 136), 0), ((67, 256), 0), ((40, 264), 0), ((41, 375), 0), ((35, 512), 16),
    ((2, 19, 520), 0), ((21, 960), 0), ((19, 1024), 0), ((18, 1032), 0), ((2, 3, 5, 2048), 0),
    ((11, 2047), 1), ((9, 2056), 0), ((7, 4096), 8), ((6, 4099), 0), ((5, 8192), 0), ((4, 8200), 0),
    ((3, 16384), 0), ((3, 16383), 2),
    # rows in pairs of values, and even ones whose stride is odd
    ((7, 2), 0), ((33, 66), 0), ((35, 300), 36), ((40, 258), 0), ((21, 962), 4), ((11, 2046), 2), ((6, 4098), 0),
    ((5, 8190), 0), ((3, 16382), 0), ((9, 66), 3),
]


@pytest.mark.parametrize("store", ["bf16", "fp32"])
@pytest.mark.parametrize("shape,pad", SHAPES)
def test_both_ways(shape, pad, store):
    x, w, b, dy, dres = make(sum(shape), shape, store, pad)
    y, stats = ringx.ringx_layer_norm(x, w, b)
    check_forward(x, w, b, store, y, stats)
    dx, dw, db = ringx.ringx_layer_norm_bwd(x, dy, stats, w, b, dres=dres)
    check_backward(x, dy, stats, w, dres, store, dx, dw, db)


@pytest.mark.parametrize("store", ["bf16", "fp32"])
@pytest.mark.parametrize("weight,bias,res", [(False, False, False), (True, False, True), (False, True, False)])
def test_without_some(store, weight, bias, res):
    x, w, b, dy, dres = make(3, (50, 96), store)
    w, b, dres = w if weight else None, b if bias else None, dres if res else None
    y, none = ringx.ringx_layer_norm(x, w, b, need_stats=False)
    assert none is None
    y2, stats = ringx.ringx_layer_norm(x, w, b)
    assert torch.equal(y, y2)
    check_forward(x, w, b, store, y, stats)
    dx, dw, db = ringx.ringx_layer_norm_bwd(x, dy, stats, w, b, dres=dres)
    assert (dw is not None) == weight and (db is not None) == bias
    check_backward(x, dy, stats, w, dres, store, dx, dw, db)


@pytest.mark.parametrize("shape,pad", [((1, 8), 0), ((33, 65), 0), ((65, 136), 0), ((41, 375), 3), ((2, 19, 520), 0),
                                       ((18, 1032), 8), ((9, 2056), 0), ((6, 4099), 0), ((4, 8200), 0),
                                       ((3, 16383), 0), ((35, 302), 0), ((18, 1034), 6), ((4, 8198), 0),
                                       ((5, 5002), 0)])
def test_gradient_in_32_bits(shape, pad):
    x, w, b, dy, dres = make(sum(shape) + 1, shape, "bf16", pad)
    dy = torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(2), device="cuda")
    _, stats = ringx.ringx_layer_norm(x, w, b)
    dx, dw, db = ringx.ringx_layer_norm_bwd(x, dy, stats, w, b, dres=dres)
    assert dx.dtype is torch.bfloat16
    check_backward(x, dy, stats, w, dres, "bf16", dx, dw, db)
    same = ringx.ringx_layer_norm_bwd(x, dy.bfloat16(), stats, w, b, dres=dres)
    wide = ringx.ringx_layer_norm_bwd(x, dy.bfloat16().float(), stats, w, b, dres=dres)
    assert all(torch.equal(p, q) for p, q in zip(same, wide))


@pytest.mark.parametrize("store,rows,C", [("bf16", 5003, 192), ("fp32", 4501, 384), ("bf16", 3001, 2048),
                                          ("fp32", 1201, 4096), ("bf16", 20011, 40), ("bf16", 1301, 3000),
                                          ("bf16", 1203, 2051), ("bf16", 1201, 4104), ("bf16", 603, 8200),
                                          ("fp32", 601, 5001), ("fp32", 401, 9001), ("bf16", 5003, 300),
                                          ("bf16", 1203, 2050)])
def test_many_rows(store, rows, C):
    # more rows than workgroups take at once, the last ones short
    x, w, b, dy, dres = make(rows, (rows, C), store)
    y, stats = ringx.ringx_layer_norm(x, w, b)
    check_forward(x, w, b, store, y, stats)
    dx, dw, db = ringx.ringx_layer_norm_bwd(x, dy, stats, w, b, dres=dres)
    check_backward(x, dy, stats, w, dres, store, dx, dw, db)
    again = ringx.ringx_layer_norm_bwd(x, dy, stats, w, b, dres=dres)
    assert all(torch.equal(p, q) for p, q in zip((dx, dw, db), again))


@pytest.mark.parametrize("store", ["bf16", "fp32"])
def test_far_from_zero(store):
    # a mean of 4000 deviations: the squares are those of the differences
    g = np.random.default_rng(9)
    x = torch.from_numpy((4096.0 + g.integers(-1, 2, (13, 300)) * 32.0).astype(np.float32)).to(DT[store]).cuda()
    y, stats = ringx.ringx_layer_norm(x)
    check_forward(x, None, None, store, y, stats)


def test_constant_rows_and_what_is_not_finite():
    x = torch.full((6, 512), 7.0, dtype=torch.bfloat16, device="cuda")
    x[1, 3] = float("inf")
    x[2, 5] = float("nan")
    y, stats = ringx.ringx_layer_norm(x, eps=1e-5)
    assert torch.isnan(y[1:3]).all()                      # a row's own, as by its formula
    ok = [0, 3, 4, 5]
    assert (y[ok] == 0).all() and (stats[0, ok] == 7).all()
    assert (stats[1, ok] - 1e-5 ** -0.5).abs().max() < 1e-3 * 1e-5 ** -0.5 * 1e-3


def test_buffers_of_the_caller_and_rows_behind():
    x, w, b, dy, dres = make(5, (30, 200), "bf16")
    wide = torch.full((40, 200), 9.0, dtype=torch.bfloat16, device="cuda")
    s = torch.empty(2, 30, device="cuda")
    y, stats = ringx.ringx_layer_norm(x, w, b, y=wide[:30], stats=s)
    assert y.data_ptr() == wide.data_ptr() and stats is s and (wide[30:] == 9).all()
    ws = torch.empty(ringx.ringx_layer_norm_bwd_workspace_bytes(30, 200, ringx.RINGX_BF16), dtype=torch.uint8,
                     device="cuda")
    out = [torch.full((40, 200), 9.0, dtype=torch.bfloat16, device="cuda")[:30],
           torch.empty(200, device="cuda"), torch.empty(200, device="cuda")]
    got = ringx.ringx_layer_norm_bwd(x, dy, s, w, b, dres=dres, dx=out[0], dweight=out[1], dbias=out[2],
                                     workspace=ws)
    assert all(p is q for p, q in zip(got, out))
    check_backward(x, dy, s, w, dres, "bf16", *got)


def test_another_stream():
    x, w, b, dy, dres = make(6, (300, 384), "bf16")
    ref = ringx.ringx_layer_norm(x, w, b)
    back = ringx.ringx_layer_norm_bwd(x, dy, ref[1], w, b, dres=dres)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    y, stats = ringx.ringx_layer_norm(x, w, b, stream=side)
    got = ringx.ringx_layer_norm_bwd(x, dy, stats, w, b, dres=dres, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(y, ref[0]) and torch.equal(stats, ref[1])
    assert all(torch.equal(p, q) for p, q in zip(got, back))


def test_two_streams_at_once_and_operands_that_are_one():
    sets = [make(i, (900 + 77 * i, 200), "bf16") for i in range(2)]

    def step(i, **kw):
        x, w, b, dy, dres = sets[i]
        y, stats = ringx.ringx_layer_norm(x, w, b, **kw)
        return (y, stats, *ringx.ringx_layer_norm_bwd(x, dy, stats, w, b, dres=dres, **kw))

    ref = [step(i) for i in range(2)]
    sides = [torch.cuda.Stream() for _ in range(2)]
    for side in sides:
        side.wait_stream(torch.cuda.current_stream())
    got = [step(i, stream=sides[i]) for _ in range(4) for i in range(2)]
    for side in sides:
        torch.cuda.current_stream().wait_stream(side)
    for k, out in enumerate(got):
        assert all(torch.equal(p, q) for p, q in zip(ref[k % 2], out))
    # inputs may be the same tensor
    x, w, b, _, _ = sets[0]
    stats = ref[0][1]
    one = ringx.ringx_layer_norm_bwd(x, x, stats, w, w, dres=x)
    two = ringx.ringx_layer_norm_bwd(x, x.clone(), stats, w.clone(), b, dres=x.clone())
    assert all(torch.equal(p, q) for p, q in zip(one, two))


def test_offsets_past_32_bits():
    rows, C = 2 ** 20 + 300, 2056      # 2.16e9 values
    g = torch.Generator(device="cuda").manual_seed(3)
    x, dres = (torch.randn(rows, C, generator=g, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    w, b = (torch.randn(C, generator=g, device="cuda") for _ in range(2))
    at = torch.cat([torch.arange(64), torch.arange(rows - 200, rows)]).cuda()
    y, stats = ringx.ringx_layer_norm(x, w, b)
    check_forward(x[at], w, b, "bf16", y[at], stats[:, at])
    # the other rows' gradients are zero, which adds nothing to the weights'
    dy = torch.zeros_like(x)
    dy[at] = torch.randn(len(at), C, generator=g, dtype=torch.bfloat16, device="cuda")
    dx, dw, db = ringx.ringx_layer_norm_bwd(x, dy, stats, w, b, dres=dres)
    check_backward(x[at], dy[at], stats[:, at], w, dres[at], "bf16", dx[at], dw, db)


def test_captured_and_replayed():
    x, w, b, dy, dres = make(7, (700, 192), "bf16")

    def step():
        y, stats = ringx.ringx_layer_norm(x, w, b)
        return (y, stats, *ringx.ringx_layer_norm_bwd(x, dy, stats, w, b, dres=dres))

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for seed in range(3):
        new = make(70 + seed, (700, 192), "bf16")
        x.copy_(new[0]), dy.copy_(new[3])
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(out, step()))


def test_gradients_are_differences():
    # the kernels' own forward in fp32 along a random direction: truncation h^2 times a third derivative of
    # order 1, rounding 2^-23 of a loss of order sqrt(values) over h
    x, w, b, dy, _ = make(8, (6, 40), "fp32")
    _, stats = ringx.ringx_layer_norm(x, w, b, eps=1e-2)
    dx, dw, db = ringx.ringx_layer_norm_bwd(x, dy, stats, w, b)
    g = torch.Generator(device="cuda").manual_seed(1)
    h = 2.0 ** -7
    for which, grad in (("x", dx), ("w", dw), ("b", db)):
        at = {"x": x, "w": w, "b": b}
        d = torch.randn(at[which].shape, generator=g, device="cuda")
        up, down = dict(at), dict(at)
        up[which], down[which] = at[which] + h * d, at[which] - h * d
        loss = [(ringx.ringx_layer_norm(p["x"], p["w"], p["b"], eps=1e-2)[0].double() * dy.double()).sum()
                for p in (up, down)]
        num = float(loss[0] - loss[1]) / (2 * h)
        size = float((grad.double() * d.double()).abs().sum())
        assert abs(num - float((grad.double() * d.double()).sum())) <= 1e-3 * size


def test_refusals():
    x, w, b, dy, dres = make(1, (8, 64), "bf16")
    _, stats = ringx.ringx_layer_norm(x, w, b)
    ln, bwd = ringx.ringx_layer_norm, ringx.ringx_layer_norm_bwd
    for bad in (lambda: ln(x.t()), lambda: ln(x[:, ::2]), lambda: ln(x, w[:63]), lambda: ln(x, w.double()),
                lambda: ln(x, w.cpu()), lambda: ln(x.half()), lambda: ln(x.cpu()),
                lambda: ln(x.view(2, 4, 64).transpose(0, 1)), lambda: ln(x, y=x.float()),
                lambda: ln(x, stats=torch.empty(2, 7, device="cuda")),
                lambda: bwd(x, dy[:4], stats, w), lambda: bwd(x, dy.double(), stats, w),
                lambda: bwd(x, dy[:4].float(), stats, w), lambda: bwd(x.float(), dy, stats, w),
                lambda: bwd(x, dy, stats[:, :4], w), lambda: bwd(x, dy, stats, w, dres=dres.float()),
                lambda: bwd(x, dy, stats, None, b, dweight=torch.empty(64, device="cuda")),
                lambda: ln(x, eps=-1.0), lambda: ln(x, eps=float("nan")), lambda: ln(x, y=x),
                lambda: bwd(x, dy, stats, w, dx=dy), lambda: ln(x[:0]),
                lambda: bwd(x, dy, stats, w, workspace=torch.empty(64, dtype=torch.uint8, device="cuda"))):
        with pytest.raises((ValueError, TypeError, ringx.RingxError)):
            bad()
