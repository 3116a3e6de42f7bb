"""The linear layer with bias, activation and residual, forward and backward, on the GPU against the fp64
oracle.

Bounds are those of rounding: a product of R terms is off by at most R + 8 steps of 2^-23 of its terms' sizes
(the matrix cores add in fp32, not necessarily to nearest); the activations by 17 E of 1 + |z|, E = 2^-24 (the
error function's 1.5e-7 / 2 = 1.3 E, the hardware's exponential and reciprocal of a step each, and the
roundings between); what is stored in bf16 by 2^-8 of it, dz among it."""

import numpy as np
import pytest
import torch

from oracle import block_fp64 as ob
from paper_2507_16697_amd import ringx

from parity_util import to_host_f64

pytestmark = pytest.mark.gpu

E, S = 2.0 ** -24, 2.0 ** -23
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}
f64 = to_host_f64


def unit(store):
    return 2.0 ** -8 if store == "bf16" else 0.0


def dev(a, store):
    return torch.from_numpy(np.asarray(a, dtype=np.float32)).to(DT[store]).cuda()


def make(seed, lead, K, O, store, heads=0, pad=0):
    """x [*lead, K] (a slice of wider rows with pad; or [B, heads, N, K / heads]), w, bias, residual, dy."""
    g = np.random.default_rng(seed)
    if heads:
        x = dev(g.standard_normal((lead[0], heads, lead[1], K // heads)), store)
    else:
        x = dev(g.standard_normal((*lead, K + pad)), store)[..., :K]
    w = dev(g.standard_normal((O, K)) * K ** -0.5, store)
    b = dev(g.standard_normal(O), "fp32")
    res, dy = (dev(g.standard_normal((*lead, O)), store) for _ in range(2))
    return x, w, b, res, dy


def check(got, ref, bound):
    err = np.abs(f64(got).reshape(ref.shape) - ref)
    assert np.isfinite(err).all() and (err <= 1.01 * bound + 1e-30).all(), float((err / (bound + 1e-30)).max())


def check_forward(x, w, b, act, res, store, y, pre):
    X, W = ob.rows(f64(x)), f64(w)
    ref, z = ob.linear(f64(x), W, None if b is None else f64(b), act, None if res is None else f64(res))
    zb = S * (X.shape[1] + 8) * (np.abs(X) @ np.abs(W).T) + E * np.abs(z)
    if pre is not None:
        check(pre, z, zb + unit(store) * np.abs(z))
    yb = zb if act == "none" else 1.13 * zb + 17 * E * (1 + np.abs(z))
    size = np.abs(ref) if res is None else np.abs(ref) + np.abs(f64(res)).reshape(ref.shape)
    check(y, ref, yb + E * size + unit(store) * np.abs(ref))


def check_backward(x, w, dy, pre, act, store, dx, dw, db, dw_unit=0.0, had=(0.0, 0.0)):
    X, W, G = ob.rows(f64(x)), f64(w), f64(dy).reshape(-1, w.shape[0])
    P = None if pre is None else f64(pre).reshape(G.shape)
    rx, rw, rb = ob.linear_bwd(f64(x), W, f64(dy), P, act)
    dz = np.abs(G) if act == "none" else np.abs(G * ob.act_grad(P, act))
    off = 0.0 if act == "none" else 17 * E * (1 + np.abs(P)) * np.abs(G) + E * dz
    cut = off if act == "none" else off + unit(store) * (dz + off)
    if dx is not None:
        b = (cut + S * (G.shape[1] + 8) * dz) @ np.abs(W) if act != "none" else \
            S * (G.shape[1] + 8) * (dz @ np.abs(W))
        u = 0.0 if dx.dtype is torch.float32 else unit(store)
        check(dx, rx, ob.unrows(b, f64(x)) + (u + E) * np.abs(rx))
    if dw is not None:
        b = S * (G.shape[0] + 8) * (dz.T @ np.abs(X))
        if act != "none":
            b = b + cut.T @ np.abs(X)
        check(dw, rw + had[0], b + dw_unit * np.abs(rw) + E * (np.abs(rw) + np.abs(had[0])))
    if db is not None:
        b = E * (G.shape[0] + 8) * dz.sum(0) + (0.0 if act == "none" else off.sum(0))
        check(db, rb + had[1], b + E * (np.abs(rb) + np.abs(had[1])))


ACTS = ["none", "gelu", "gelu_tanh", "silu"]
SHAPES = [
    # lead, K, O, heads, pad
    ((1,), 8, 8, 0, 0), ((1,), 64, 16, 0, 0), ((3,), 200, 40, 0, 8), ((16,), 512, 130, 0, 0),
    ((17,), 72, 33, 0, 0), ((2, 16), 1000, 64, 0, 0), ((64,), 136, 200, 0, 16), ((65,), 64, 64, 0, 0),
    ((2, 45), 8, 24, 0, 0), ((129,), 192, 128, 0, 0), ((130,), 200, 136, 0, 24), ((257,), 264, 120, 0, 0),
    # a few rows: blocks of 16 of them, two blocks of features at a time, ends of both and of K
    ((20,), 72, 8200, 0, 0), ((40,), 1032, 8210, 0, 0), ((60,), 200, 8192, 0, 8), ((45,), 200, 4100, 0, 0), ((33,), 72, 4096, 0, 0),
    ((48,), 1096, 40, 0, 0), ((2, 20), 192, 72, 3, 0),
    # the bias's gradient beside the products, and before them
    ((700,), 64, 40, 0, 0), ((1024,), 64, 64, 0, 0), ((1025,), 64, 64, 0, 0),
    # widths and rows that fit no 16-byte piece
    ((1,), 1, 1, 0, 0), ((5,), 7, 3, 0, 0), ((77,), 375, 96, 0, 0), ((70,), 33, 129, 0, 5),
    ((131,), 64, 131, 0, 3), ((200,), 129, 65, 0, 0),
    # an attention's layout: heads that the products walk themselves, and others
    ((2, 64), 128, 64, 2, 0), ((2, 33), 192, 72, 3, 0), ((1, 128), 256, 130, 2, 0), ((3, 50), 120, 40, 5, 0),
    ((2, 3), 128, 48, 2, 0), ((2, 70), 42, 30, 3, 0), ((1, 192), 64, 64, 1, 0),
]


@pytest.mark.parametrize("store", ["bf16", "fp32"])
@pytest.mark.parametrize("lead,K,O,heads,pad", SHAPES)
def test_both_ways(lead, K, O, heads, pad, store):
    x, w, b, res, dy = make(K + O, lead, K, O, store, heads, pad)
    act = ACTS[(K + O) % 4]
    y, pre = ringx.ringx_linear(x, w, b, act=act, residual=res, need_pre=True)
    assert y.shape == (*lead, O)
    check_forward(x, w, b, act, res, store, y, pre)
    kept = None if act == "none" else pre
    dx, dw, db = ringx.ringx_linear_bwd(x, w, dy, pre=kept, act=act, bias=b)
    assert dx.shape == x.shape and dw.dtype is torch.float32
    check_backward(x, w, dy, kept, act, store, dx, dw, db)


@pytest.mark.parametrize("store", ["bf16", "fp32"])
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("M,K,O", [(9, 96, 50), (150, 128, 72)])
def test_activations_over_their_range(M, K, O, act, store):
    x, w, b, _, dy = make(4, (M,), K, O, store)
    x = x * 12.0
    y, pre = ringx.ringx_linear(x, w, b, act=act, need_pre=True)
    check_forward(x, w, b, act, None, store, y, pre)
    kept = None if act == "none" else pre
    check_backward(x, w, dy, kept, act, store, *ringx.ringx_linear_bwd(x, w, dy, pre=kept, act=act, bias=b))


@pytest.mark.parametrize("act", ["gelu", "gelu_tanh", "silu"])
def test_activations_at_their_ends(act):
    # far out, where the factors are 0 and infinity
    z = torch.tensor([-3e38, -1e20, -200.0, -40.0, 0.0, 40.0, 200.0, 1e20, 3e38], device="cuda")
    w, x = torch.zeros(9, 4, device="cuda"), torch.zeros(70, 4, device="cuda")
    y, pre = ringx.ringx_linear(x, w, z, act=act, need_pre=True)
    assert torch.equal(pre[0], z)
    want = torch.where(z > 0, z, torch.zeros_like(z))
    assert (y[3] - want).abs().max() <= 1e-15      # silu(-40) is -2e-16
    dy = torch.ones(70, 9, device="cuda")
    dx, dw, db = ringx.ringx_linear_bwd(x, w, dy, pre=pre, act=act, bias=z)
    slope = torch.tensor([0.0, 0, 0, 0, 0.5, 1, 1, 1, 1], device="cuda")
    # 70 sums of 1, each to 17 E (1 + |z|) where |z| is at most 40
    assert (db - 70 * slope).abs().max() <= 70 * (17 * 41 + 70) * E


@pytest.mark.parametrize("store", ["bf16", "fp32"])
@pytest.mark.parametrize("M,K,O,heads", [
    (4100, 384, 1152, 0),      # parts of r along the weights' gradient
    (4097, 328, 3848, 0),      # large tiles, ragged
    (8194, 1032, 520, 0),      # last tiles in parts
    (5000, 250, 60, 0),        # rows copied
    (4608, 512, 768, 8),       # heads of 64, batches of whole steps
    (1000, 520, 264, 0),       # both gradients in one launch, two groups of waves
    (3000, 712, 392, 0),       # and one group
    (70, 4096, 96, 0),         # parts of r forward
    (300, 2072, 200, 0),
    (1500, 301, 1100, 0),      # fp32: tiles of 64 forward
    (1500, 1501, 700, 0),      # and of both gradients in one launch
    (2100, 1601, 1400, 0),     # and of each by itself
    (8190, 1101, 8200, 0),     # tiles of 128, ragged
    (4000, 601, 302, 0),       # tiles of 64 and of 32 in one backward
    (9000, 1001, 130, 0),      # of 128 and of 32
])
def test_large(M, K, O, heads, store):
    lead = (2, M // 2) if heads else (M,)
    x, w, b, res, dy = make(M, lead, K, O, store, heads)
    y, pre = ringx.ringx_linear(x, w, b, act="gelu", residual=res, need_pre=True)
    dx, dw, db = ringx.ringx_linear_bwd(x, w, dy, pre=pre, act="gelu", bias=b)
    again = ringx.ringx_linear_bwd(x, w, dy, pre=pre, act="gelu", bias=b)
    assert all(torch.equal(p, q) for p, q in zip((dx, dw, db), again))
    assert torch.equal(y, ringx.ringx_linear(x, w, b, act="gelu", residual=res)[0])
    X, W, G, P = (t.double() for t in (x, w, dy.reshape(-1, O), pre.reshape(-1, O)))
    X = X.transpose(1, 2).reshape(-1, K) if heads else X
    # in 64 bits on the GPU, whole; the bounds of the module's note with the sums' sizes
    z = X @ W.t() + b.double()
    phi = torch.special.ndtr(z)
    ref = z * phi + res.double().reshape(-1, O)
    zb = S * (K + 8) * (X.abs() @ W.abs().t()) + E * z.abs()
    u = unit(store)
    yb = 1.13 * zb + 17 * E * (1 + z.abs()) + (u + E) * ref.abs() + E * res.double().abs().reshape(-1, O)
    assert ((y.double().reshape(-1, O) - ref).abs() <= 1.01 * yb).all()
    assert ((pre.double().reshape(-1, O) - z).abs() <= 1.01 * (zb + u * z.abs())).all()
    slope = torch.special.ndtr(P) + P * torch.exp(-P * P / 2) / np.sqrt(2 * np.pi)
    dz = G * slope
    off = 17 * E * (1 + P.abs()) * G.abs() + (E + u) * dz.abs()
    rx = dz @ W
    xb = (off + S * (O + 8) * dz.abs()) @ W.abs() + u * rx.abs()
    gx = dx.double().transpose(1, 2).reshape(-1, K) if heads else dx.double()
    assert ((gx - rx).abs() <= 1.01 * xb).all()
    rw = dz.t() @ X
    assert ((dw.double() - rw).abs() <= 1.01 * ((off + S * (M + 8) * dz.abs()).t() @ X.abs())).all()
    assert ((db.double() - dz.sum(0)).abs() <= 1.01 * (off.sum(0) + E * (M + 8) * dz.abs().sum(0))).all()


@pytest.mark.parametrize("M,K,O", [(5, 64, 48), (300, 96, 64), (90, 41, 23)])
def test_gradients_in_parts_and_types(M, K, O):
    x, w, b, _, dy = make(2, (M,), K, O, "bf16")
    whole = ringx.ringx_linear_bwd(x, w, dy, bias=b)
    dx, none, no_bias = ringx.ringx_linear_bwd(x, w, dy, need_dw=False)
    assert none is None and no_bias is None and torch.equal(dx, whole[0])
    none, dw, db = ringx.ringx_linear_bwd(x, w, dy, bias=b, need_dx=False, dw_dtype=torch.bfloat16)
    assert none is None and torch.equal(dw, whole[1].to(torch.bfloat16)) and torch.equal(db, whole[2])
    wide, _, _ = ringx.ringx_linear_bwd(x, w, dy, need_dw=False, dx_dtype=torch.float32)
    assert wide.dtype is torch.float32 and torch.equal(wide.to(torch.bfloat16), whole[0])
    check_backward(x, w, dy, None, "none", "fp32", wide, None, None)
    both = ringx.ringx_linear_bwd(x, w, dy, bias=b, dx=torch.empty_like(wide))
    assert torch.equal(both[0], wide) and torch.equal(both[1], whole[1])
    none, none2, db = ringx.ringx_linear_bwd(x, w, dy, bias=b, need_dx=False, need_dw=False)
    assert none is None and none2 is None and torch.equal(db, whole[2])
    # added to
    base = [torch.randn(O, K, device="cuda"), torch.randn(O, device="cuda")]
    got = ringx.ringx_linear_bwd(x, w, dy, bias=b, dw=base[0].clone(), dbias=base[1].clone(), accumulate_dw=True)
    check_backward(x, w, dy, None, "none", "bf16", *got, had=tuple(f64(t) for t in base))
    new = ringx.ringx_linear_bwd(x, w, dy, bias=b, accumulate_dw=True)
    assert torch.equal(new[1], whole[1]) and torch.equal(new[2], whole[2])


@pytest.mark.parametrize("store", ["bf16", "fp32"])
@pytest.mark.parametrize("M,K", [(3, 100), (140, 72), (140, 101)])
def test_what_is_not_finite_stays_in_its_row(M, K, store):
    # infinities and NaN reach the rows and features that they belong to, no padding, no neighbour
    x, w, b, _, dy = make(6, (M,), K, 40, store)
    x[1, K - 1], x[2, 0] = float("inf"), float("nan")
    w[7, K - 1] = float("nan")
    y, _ = ringx.ringx_linear(x, w, b)
    bad = ~torch.isfinite(y)
    want = torch.zeros_like(bad)
    want[1:3], want[:, 7] = True, True
    assert torch.equal(bad, want)
    x, w, b, _, dy = make(6, (M,), K, 40, store)
    dy[M - 1, 39] = float("inf")
    dx, dw, db = ringx.ringx_linear_bwd(x, w, dy, bias=b)
    assert not torch.isfinite(dx[M - 1]).any() and torch.isfinite(dx[:M - 1]).all()
    assert not torch.isfinite(dw[39]).any() and torch.isfinite(dw[:39]).all()
    assert not torch.isfinite(db[39]) and torch.isfinite(db[:39]).all()


def test_memory_behind_the_operands_is_not_read_into_the_result():
    # the tensors are slices of larger ones that hold NaN around them
    for M, K, O in ((70, 40, 24), (70, 39, 23), (5, 40, 24), (300, 136, 200)):
        x, w, _, _, dy = make(M, (M,), K, O, "bf16")

        def inside(t):
            n = t.numel()
            big = torch.full((n + 4096,), float("nan"), dtype=t.dtype, device="cuda")
            big[2048:2048 + n] = t.flatten()
            return big[2048:2048 + n].view(t.shape)

        ref = (ringx.ringx_linear(x, w)[0], *ringx.ringx_linear_bwd(x, w, dy)[:2])
        x, w, dy = inside(x), inside(w), inside(dy)
        got = (ringx.ringx_linear(x, w)[0], *ringx.ringx_linear_bwd(x, w, dy)[:2])
        assert all(torch.equal(p, q) for p, q in zip(ref, got))


def test_buffers_of_the_caller_and_rows_behind():
    x, w, b, res, dy = make(5, (100,), 64, 72, "bf16")
    wide = torch.full((130, 72), 9.0, dtype=torch.bfloat16, device="cuda")
    kept = torch.full((130, 72), 9.0, dtype=torch.bfloat16, device="cuda")
    y, pre = ringx.ringx_linear(x, w, b, act="silu", residual=res, y=wide[:100], pre=kept[:100])
    assert (wide[100:] == 9).all() and (kept[100:] == 9).all()
    check_forward(x, w, b, "silu", res, "bf16", y, pre)
    out = torch.full((130, 64), 9.0, dtype=torch.bfloat16, device="cuda")
    grad = torch.full((80, 64), 9.0, device="cuda")
    dx, dw, _ = ringx.ringx_linear_bwd(x, w, dy, pre=pre, act="silu", dx=out[:100], dw=grad[:72])
    assert (out[100:] == 9).all() and (grad[72:] == 9).all()
    check_backward(x, w, dy, pre, "silu", "bf16", dx, dw, None)


def test_another_stream_and_its_workspace():
    x, w, b, res, dy = make(6, (333,), 250, 96, "bf16")

    def step(**kw):
        y, pre = ringx.ringx_linear(x, w, b, act="gelu", residual=res, need_pre=True, **kw)
        return (y, pre, *ringx.ringx_linear_bwd(x, w, dy, pre=pre, act="gelu", bias=b, **kw))

    ref = step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = step(stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(p, q) for p, q in zip(ref, got))


def test_two_streams_at_once_and_operands_that_are_one():
    sets = [make(i, (500 + 77 * i,), 136, 200, "bf16") for i in range(2)]

    def step(i, **kw):
        x, w, b, res, dy = sets[i]
        y, pre = ringx.ringx_linear(x, w, b, act="silu", residual=res, need_pre=True, **kw)
        return (y, pre, *ringx.ringx_linear_bwd(x, w, dy, pre=pre, act="silu", bias=b, **kw))

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
    t = sets[0][0][:136].contiguous()
    a, b, c = t.clone(), t.clone(), t.clone()
    assert torch.equal(ringx.ringx_linear(t, t, residual=t)[0], ringx.ringx_linear(a, b, residual=c)[0])
    one = ringx.ringx_linear_bwd(t, t, t, pre=t, act="gelu")
    two = ringx.ringx_linear_bwd(a, b, c, pre=t, act="gelu")
    assert all(torch.equal(p, q) for p, q in zip(one[:2], two[:2]))


def ends(M):
    return torch.cat([torch.arange(64), torch.arange(M - 200, M)]).cuda()


@pytest.mark.parametrize("K,O", [(16, 4104), (4104, 16)])
def test_offsets_past_32_bits(K, O):
    M = 2 ** 19 + 300     # times 4104: 2.15e9 values
    g = torch.Generator(device="cuda").manual_seed(3)
    rnd = lambda *n: torch.randn(*n, generator=g, dtype=torch.bfloat16, device="cuda")   # noqa: E731
    x, w, b, res = rnd(M, K), rnd(O, K), rnd(O).float(), rnd(M, O)
    at = ends(M)
    y, pre = ringx.ringx_linear(x, w, b, act="gelu", residual=res, need_pre=True)
    check_forward(x[at], w, b, "gelu", res[at], "bf16", y[at], pre[at])
    # the other rows' gradients are zero, which adds nothing to any sum
    dy = torch.zeros_like(y)
    dy[at] = rnd(len(at), O)
    dx, dw, db = ringx.ringx_linear_bwd(x, w, dy, pre=pre, act="gelu", bias=b)
    check_backward(x[at], w, dy[at], pre[at], "gelu", "bf16", dx[at], dw, db)


@pytest.mark.parametrize("store,M,step", [("bf16", 1100, 2 ** 21 - 8), ("bf16", 1100, 2 ** 21 + 8),
                                          ("bf16", 40, 2 ** 26), ("fp32", 1030, 2 ** 21)])
def test_rows_far_apart(store, M, step):
    K, O = 64, 72
    x, w, b, res, dy = make(3, (M,), K, O, store)
    far = torch.empty(M * step, dtype=x.dtype, device="cuda").as_strided((M, K), (step, 1))
    far.copy_(x)
    y, pre = ringx.ringx_linear(far, w, b, act="silu", residual=res, need_pre=True)
    check_forward(x, w, b, "silu", res, store, y, pre)
    dx, dw, db = ringx.ringx_linear_bwd(far, w, dy, pre=pre, act="silu", bias=b)
    check_backward(x, w, dy, pre, "silu", store, dx, dw, db)


@pytest.mark.parametrize("M", [2, 70])
@pytest.mark.parametrize("K,O", [(2 ** 20, 5), (5, 2 ** 20)])
def test_widest(K, O, M):
    x, w, b, _, dy = make(4, (M,), K, O, "bf16")
    y, _ = ringx.ringx_linear(x, w, b)
    check_forward(x, w, b, "none", None, "bf16", y, None)
    check_backward(x, w, dy, None, "none", "bf16", *ringx.ringx_linear_bwd(x, w, dy, bias=b))


def test_captured_and_replayed():
    shapes = [((7,), 128, 64), ((150,), 250, 96), ((2000,), 64, 64)]
    sets = [make(i, *s, "bf16") for i, s in enumerate(shapes)]

    def step():
        out = []
        for x, w, b, res, dy in sets:
            y, pre = ringx.ringx_linear(x, w, b, act="gelu", residual=res, need_pre=True)
            out += [y, pre, *ringx.ringx_linear_bwd(x, w, dy, pre=pre, act="gelu", bias=b)]
        return out

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for seed in range(3):
        for i, s in enumerate(shapes):
            new = make(100 * seed + i, *s, "bf16")
            sets[i][0].copy_(new[0]), sets[i][4].copy_(new[4])
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(out, step()))


@pytest.mark.parametrize("act", ACTS)
def test_gradients_are_differences(act):
    x, w, b, _, dy = make(8, (70,), 24, 16, "fp32")
    _, pre = ringx.ringx_linear(x, w, b, act=act, need_pre=True)
    dx, dw, db = ringx.ringx_linear_bwd(x, w, dy, pre=None if act == "none" else pre, act=act, bias=b)
    g = torch.Generator(device="cuda").manual_seed(1)
    h = 2.0 ** -7      # truncation h^2 of a third derivative of order 1, rounding 2^-23 / h
    for which, grad in (("x", dx), ("w", dw), ("b", db)):
        at = {"x": x, "w": w, "b": b}
        d = torch.randn(at[which].shape, generator=g, device="cuda")
        up, down = dict(at), dict(at)
        up[which], down[which] = at[which] + h * d, at[which] - h * d
        loss = [(ringx.ringx_linear(p["x"], p["w"], p["b"], act=act)[0].double() * dy.double()).sum()
                for p in (up, down)]
        num = float(loss[0] - loss[1]) / (2 * h)
        size = float((grad.double() * d.double()).abs().sum())
        assert abs(num - float((grad.double() * d.double()).sum())) <= 1e-3 * size


def test_refusals():
    x, w, b, res, dy = make(1, (8,), 64, 48, "bf16")
    lin, bwd = ringx.ringx_linear, ringx.ringx_linear_bwd
    x4 = torch.zeros(2, 2, 8, 32, dtype=torch.bfloat16, device="cuda")
    for bad in (lambda: lin(x, w[:, :32]), lambda: lin(x, w.float()), lambda: lin(x, w.t()), lambda: lin(x, w[0]),
                lambda: lin(x, w, b[:4]), lambda: lin(x, w, b.to(torch.bfloat16)), lambda: lin(x, w, act="relu6"),
                lambda: lin(x, w, residual=res[:4]), lambda: lin(x, w, residual=res.float()),
                lambda: lin(x.t(), w), lambda: lin(x.cpu(), w), lambda: lin(x, w.cpu()), lambda: lin(x[:0], w),
                lambda: lin(x, w, y=res, residual=res), lambda: lin(x, w, y=x), lambda: lin(x4.transpose(1, 2), w),
                lambda: lin(x4[..., :16], w), lambda: bwd(x, w, dy[:4]), lambda: bwd(x, w, dy.float()),
                lambda: bwd(x, w, dy, act="gelu"), lambda: bwd(x, w, dy, pre=dy), lambda: bwd(x, w, dy, dx=x),
                lambda: bwd(x, w, dy, dx_dtype=torch.float16),
                lambda: bwd(x4, w, dy.view(2, 4, 48)), lambda: bwd(x, w, dy, dw_dtype=torch.float16),
                lambda: bwd(x, w, dy, dw=w),
                lambda: bwd(x, w, dy, need_dx=False, need_dw=False),
                lambda: bwd(x, w, dy, dw_dtype=torch.bfloat16, accumulate_dw=True),
                lambda: bwd(x, w, dy, dbias=torch.zeros(48, device="cuda")),
                lambda: bwd(x, w, dy, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))):
        with pytest.raises((ValueError, TypeError, ringx.RingxError)):
            bad()
