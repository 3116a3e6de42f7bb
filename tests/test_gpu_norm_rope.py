"""The per-head norm of queries and keys with their rotation, both directions, on the GPU against the
fp64 oracle, and one block's training step of all parts together.

Bounds are those of rounding: fp32 sums and products, sine and cosine within 2 steps of an angle that
is held to 2^-25 of a turn, one rounding to the stored type."""

import numpy as np
import pytest
import torch

from oracle import dropout_fp64 as od
from oracle import norm_rope_fp64 as on
from paper_2507_16697_amd import ringx

from parity_util import to_host_f64
from test_gpu_dropout import SEED, bounds, state

pytestmark = pytest.mark.gpu

E = 2.0 ** -24
# an angle's 2^-25 of a turn is 2 pi 2^-25 radians; the sine's own error and the products' beside it
TURN = 2 * np.pi * 2.0 ** -25 + 8 * E


def unit(store):
    return 2.0 ** -8 if store == "bf16" else 0.0


def make(seed, B, N, H, Hkv, d, rot, store, weights=True, pos="grid", pad=0, std=1.0):
    """Device arguments and their exact fp64 values."""
    g = np.random.default_rng(seed)
    dt = torch.float32 if store == "fp32" else torch.bfloat16
    cols = (H + 2 * Hkv) * d
    wide = torch.from_numpy((g.standard_normal((B, N, cols + pad)) * std).astype(np.float32)).to(dt).cuda()
    a = {"qkv": wide[:, :, :cols], "freqs": None, "rot": rot, "pos": None, "pos0": 0, "qw": None,
         "kw": None}
    f = np.concatenate([10000.0 ** (-np.arange(0, r, 2) / max(r, 1)) for r in rot])
    a["freqs"] = torch.from_numpy(f).cuda()
    if pos == "grid":
        a["pos"] = torch.from_numpy(g.integers(0, 4096, (N, len(rot)), dtype=np.int32)).cuda()
    elif pos == "batch":
        a["pos"] = torch.from_numpy(g.integers(-2 ** 31, 2 ** 31, (B, N, len(rot)),
                                               dtype=np.int32)).cuda()
    else:
        a["pos0"] = pos
    if weights:
        a["qw"], a["kw"] = (torch.from_numpy(g.uniform(-1.5, 1.5, d).astype(np.float32)).cuda()
                            for _ in range(2))
    return a, exact_of(a)


def exact_of(a):
    x = {"qkv": to_host_f64(a["qkv"]), "freqs": a["freqs"].cpu().numpy(), "rot": a["rot"],
         "pos": None if a["pos"] is None else a["pos"].cpu().numpy(), "pos0": a["pos0"]}
    for w in ("qw", "kw"):
        x[w] = None if a[w] is None else to_host_f64(a[w])
    return x


def forward(a, H, Hkv, **kw):
    return ringx.ringx_qkv_norm_rope(a["qkv"], H, Hkv, a["freqs"], a["rot"], pos=a["pos"],
                                     pos0=a["pos0"], q_weight=a["qw"], k_weight=a["kw"], **kw)


def backward(a, dq, dk, dv, **kw):
    return ringx.ringx_qkv_norm_rope_bwd(a["qkv"], dq, dk, dv, a["freqs"], a["rot"], pos=a["pos"],
                                         pos0=a["pos0"], q_weight=a["qw"], k_weight=a["kw"], **kw)


def mates(y, rot):
    """|y| of a dim and of the other of its pair, added (an unrotated dim: its own)."""
    y = np.abs(y)
    z, o = y.copy(), 0
    for r in rot:
        n = r // 2
        both = y[..., o:o + n] + y[..., o + n:o + 2 * n]
        z[..., o:o + n] = z[..., o + n:o + 2 * n] = both
        o += 2 * n
    return z


def angle_noise(x):
    """Error of an angle of far positions in 64 bits: three roundings of its turns, in radians."""
    top = abs(x["pos0"]) + x["qkv"].shape[1]
    if x["pos"] is not None:
        top = float(np.abs(x["pos"].astype(np.float64)).max()) + 1
    return 3 * 2.0 ** -53 * top * float(np.abs(x["freqs"]).max() if len(x["freqs"]) else 0)


def check_forward(x, H, Hkv, store, q, k, v, eps=1e-6):
    d = q.shape[-1]
    rq, rk, rv = on.qkv_norm_rope(x["qkv"], H, Hkv, x["freqs"], x["rot"], x["pos"], x["pos0"], x["qw"],
                                  x["kw"], eps)
    assert np.array_equal(to_host_f64(v), rv)
    yq, yk, _ = on.qkv_norm_rope(x["qkv"], H, Hkv, np.zeros(0), (), None, 0, x["qw"], x["kw"], eps)
    rel = (d / 2 + 12) * E + TURN + angle_noise(x)
    for got, ref, y in ((q, rq, yq), (k, rk, yk)):
        err = np.abs(to_host_f64(got) - ref)
        b = rel * mates(y, x["rot"]) + unit(store) * np.abs(ref) + 1e-30
        assert np.isfinite(err).all() and (err <= 1.01 * b).all(), float((err - b).max())


def check_backward(x, H, Hkv, store, grads, dx, dqw, dkw, eps=1e-6):
    d = grads[0].shape[-1]
    g64 = [to_host_f64(t) for t in grads]
    rx, rqw, rkw = on.qkv_norm_rope_bwd(x["qkv"], *g64, x["freqs"], x["rot"], x["pos"], x["pos0"],
                                        x["qw"], x["kw"], eps)
    heads = np.split(x["qkv"].reshape(*x["qkv"].shape[:2], H + 2 * Hkv, d).transpose(0, 2, 1, 3),
                     [H, H + Hkv], axis=1)
    rel = (2 * d + 40) * E + TURN + angle_noise(x)
    parts = []
    for y, g, w, ref, got in ((heads[0], g64[0], x["qw"], rqw, dqw), (heads[1], g64[1], x["kw"], rkw, dkw)):
        r = 1 / np.sqrt((y * y).mean(-1, keepdims=True) + eps)
        a = mates(g, x["rot"])                       # a bound of the turned gradient
        n = y.shape[0] * y.shape[1] * y.shape[2]
        if w is None:
            assert got is None
        else:
            b = (rel + (n + 64) * E) * (a * np.abs(y) * r).sum((0, 1, 2))
            assert (np.abs(to_host_f64(got) - ref) <= 1.01 * b + 1e-30).all()
            a = a * np.abs(w)
        parts.append(rel * r * (a + np.abs(y) * r * (a * np.abs(y) * r).mean(-1, keepdims=True)))
    parts.append(np.zeros_like(g64[2]))
    b = np.concatenate(parts, 1).transpose(0, 2, 1, 3).reshape(rx.shape) + unit(store) * np.abs(rx)
    err = np.abs(to_host_f64(dx) - rx)
    assert np.isfinite(err).all() and (err <= 1.01 * b + 1e-30).all(), float((err - b).max())


def grads_of(seed, B, N, H, Hkv, d):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return [torch.randn((B, h, N, d), generator=g, device="cuda") for h in (H, Hkv, Hkv)]


CASES = [
    # bf16: one token, odd counts, every head size; sections of odd halves, of part of the head, of none
    ("bf16", 1, 1, 1, 1, 64, (64,), True, 0, 0), ("bf16", 1, 1, 16, 16, 128, (128,), True, 98304, 0),
    ("bf16", 3, 37, 6, 2, 64, (20, 22, 22), True, "grid", 64), ("bf16", 2, 130, 4, 4, 128, (40, 44, 44), True, "batch", 0),
    ("bf16", 1, 65, 3, 1, 128, (2, 0, 6), False, "grid", 8), ("bf16", 1, 9, 2, 1, 64, (0,), True, 5, 0),
    ("bf16", 2, 700, 2, 2, 64, (48,), False, -1000, 0), ("bf16", 1, 4100, 8, 2, 128, (32, 48, 48), True, "grid", 0),
    # fp32: head dims on both sides of every lane count, rows that are no multiple of 16 bytes
    ("fp32", 1, 5, 2, 2, 1, (0,), True, 0, 0), ("fp32", 2, 33, 2, 1, 2, (2,), True, 0, 1),
    ("fp32", 1, 40, 3, 3, 7, (4, 2), True, "grid", 0), ("fp32", 2, 31, 4, 2, 12, (4, 4, 4), True, "batch", 3),
    ("fp32", 1, 50, 2, 2, 33, (32,), False, 2 ** 40 - 50, 0), ("fp32", 3, 151, 3, 3, 100, (30, 34, 34), True, "grid", 36),
    ("fp32", 1, 70, 1, 1, 127, (126,), True, 7, 0), ("fp32", 1, 300, 4, 2, 128, (128,), True, "batch", 2),
    ("fp32", 2, 33, 2, 2, 16, (16,), True, 11, 4), ("fp32", 1, 40, 2, 2, 32, (10, 12, 10), True, "grid", 0)]


@pytest.mark.parametrize("store,B,N,H,Hkv,d,rot,weights,pos,pad", CASES)
def test_both_directions(store, B, N, H, Hkv, d, rot, weights, pos, pad):
    print(f"norm rope {store} B={B} N={N} H={H}/{Hkv} d={d} rot={rot} pos={pos} pad={pad}", flush=True)
    a, x = make(N + d, B, N, H, Hkv, d, rot, store, weights, pos, pad)
    if len(rot) == 1 and isinstance(pos, int):
        assert a["pos"] is None
    check_forward(x, H, Hkv, store, *forward(a, H, Hkv))
    g = grads_of(N, B, N, H, Hkv, d)
    check_backward(x, H, Hkv, store, g, *backward(a, *g))


def test_rows_of_zeros_and_of_large_values():
    a, _ = make(1, 1, 12, 2, 2, 64, (64,), "bf16", pos=3)
    a["qkv"][:, 3] = 0
    a["qkv"][:, 4] *= 1e15
    a["qkv"][:, 5] *= 1e-15
    x = exact_of(a)
    check_forward(x, 2, 2, "bf16", *forward(a, 2, 2))
    g = grads_of(2, 1, 12, 2, 2, 64)
    check_backward(x, 2, 2, "bf16", g, *backward(a, *g))


def test_only_one_weight():
    a, _ = make(2, 2, 40, 4, 2, 64, (32,), "bf16", pos=0)
    a["qw"] = None
    x = exact_of(a)
    check_forward(x, 4, 2, "bf16", *forward(a, 4, 2))
    g = grads_of(3, 2, 40, 4, 2, 64)
    check_backward(x, 4, 2, "bf16", g, *backward(a, *g))


@pytest.mark.parametrize("store,d", [("bf16", 128), ("fp32", 50)])
def test_strides(store, d):
    """A batch-second layout, every other token, and one row for the whole batch."""
    H, Hkv, B, N = 2, 1, 3, 20
    a, x = make(4, B, N, H, Hkv, d, (d // 4 * 2,), store, pos=1)
    want = forward(a, H, Hkv)
    swapped = dict(a, qkv=a["qkv"].transpose(0, 1).contiguous().transpose(0, 1))
    assert swapped["qkv"].stride() != a["qkv"].stride()
    assert all(torch.equal(u, w) for u, w in zip(want, forward(swapped, H, Hkv)))
    two = torch.stack([a["qkv"], torch.full_like(a["qkv"], float("nan"))], 2).reshape(B, 2 * N, -1)
    assert all(torch.equal(u, w) for u, w in zip(want, forward(dict(a, qkv=two[:, ::2]), H, Hkv)))
    g = grads_of(5, B, N, H, Hkv, d)
    for u, w in zip(backward(a, *g), backward(dict(a, qkv=two[:, ::2]), *g)):
        assert torch.equal(u, w)
    row = a["qkv"][:1].expand(B, N, -1)
    q = forward(dict(a, qkv=row), H, Hkv)[0]
    assert all(torch.equal(q[b], want[0][0]) for b in range(B))


@pytest.mark.parametrize("store,H,d,N", [("bf16", 1, 64, 500_017), ("bf16", 1, 128, 250_009),
                                         ("fp32", 2, 32, 375_013)])
def test_large_calls_are_their_parts(store, H, d, N):
    """Calls whose tensors outgrow the caches, by another form of the kernels, against calls on parts of
    their tokens: every row to the bit, the weights' gradients to the rounding of their sums."""
    gen = torch.Generator(device="cuda").manual_seed(d)
    dt = torch.float32 if store == "fp32" else torch.bfloat16
    new = lambda *shape: torch.randn(shape, generator=gen, device="cuda")   # noqa: E731
    a = {"qkv": new(1, N, (H + 2) * d).to(dt), "rot": (d // 2,), "pos": None, "pos0": -1000,
         "freqs": torch.from_numpy(10000.0 ** (-np.arange(0, d // 2, 2) / (d // 2))).cuda(),
         "qw": 1 + 0.2 * new(d), "kw": 1 + 0.2 * new(d)}
    g = [new(1, h, N, d) for h in (H, 1, 1)]
    whole, wholeg = forward(a, H, 1), backward(a, *g)
    sums = [torch.zeros(d, dtype=torch.float64, device="cuda") for _ in range(2)]
    size = [torch.zeros(d, dtype=torch.float64, device="cuda") for _ in range(2)]
    for lo in range(0, N, 100_000):
        hi = min(N, lo + 100_000)
        part = dict(a, qkv=a["qkv"][:, lo:hi].contiguous(), pos0=lo - 1000)
        for t, u in zip(whole, forward(part, H, 1)):
            assert torch.equal(t[:, :, lo:hi], u)
        dx, dqw, dkw = backward(part, *(t[:, :, lo:hi].contiguous() for t in g))
        assert torch.equal(wholeg[0][:, lo:hi], dx)
        for i, t in enumerate((dqw, dkw)):
            sums[i] += t.double()
            # |g| |x r| summed: at most 6 standard deviations of a gradient and of a normed row each
            size[i] += 36.0 * (hi - lo) * (H if i == 0 else 1)
    for i in range(2):
        # up to 2048 workgroups' chains of N H / 8192 rows and then the parts' sums, on both sides
        steps = 2 * (N * H / 8192 + 2048 / 32 + 64)
        assert bool(((wholeg[1 + i].double() - sums[i]).abs() <= steps * E * size[i]).all())


def test_buffers_behind_the_last_row_stay():
    a, _ = make(6, 1, 37, 2, 2, 64, (64,), "bf16", pos=0)
    n = 37 * 64
    buf = torch.full((3, 2 * n + 256), 7.0, dtype=torch.bfloat16, device="cuda")
    q, k, v = (b[:2 * n].view(1, 2, 37, 64) for b in buf)
    want = forward(a, 2, 2)
    forward(a, 2, 2, q=q, k=k, v=v)
    assert all(torch.equal(u, w) for u, w in zip(want, (q, k, v)))
    assert bool((buf[:, 2 * n:] == 7).all())


def test_repeats_bitwise_and_replays():
    a, _ = make(7, 2, 600, 4, 2, 128, (40, 44, 44), "bf16")
    g = grads_of(8, 2, 600, 4, 2, 128)
    want, wantg = forward(a, 4, 2), backward(a, *g)
    q, k, v = (torch.empty_like(t) for t in want)
    dx, dqw, dkw = (torch.empty_like(t) for t in wantg)
    ws = torch.empty(ringx.ringx_qkv_norm_rope_bwd_workspace_bytes(2, 600, 4, 2, 128, ringx.RINGX_BF16),
                     dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        forward(a, 4, 2, q=q, k=k, v=v)
        backward(a, *g, dqkv=dx, dq_weight=dqw, dk_weight=dkw, workspace=ws)
    for _ in range(3):
        for t in (q, k, v, dx, dqw, dkw):
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        for u, w in zip((q, k, v, dx, dqw, dkw), want + wantg):
            assert torch.equal(u, w)
        assert all(torch.equal(u, w) for u, w in zip(backward(a, *g), wantg))


def test_binding_refusals():
    a, _ = make(9, 1, 10, 2, 2, 64, (20, 22, 22), "bf16")
    with pytest.raises(ValueError, match="freqs: shape"):
        ringx.ringx_qkv_norm_rope(a["qkv"], 2, 2, a["freqs"], (20, 22), pos=a["pos"])
    with pytest.raises(ValueError, match="pos"):
        ringx.ringx_qkv_norm_rope(a["qkv"], 2, 2, a["freqs"], a["rot"])
    with pytest.raises(TypeError, match="pos: dtype"):
        ringx.ringx_qkv_norm_rope(a["qkv"], 2, 2, a["freqs"], a["rot"], pos=a["pos"].long())
    with pytest.raises(TypeError, match="freqs: dtype"):
        ringx.ringx_qkv_norm_rope(a["qkv"], 2, 2, a["freqs"].float(), a["rot"], pos=a["pos"])
    with pytest.raises(ValueError, match="columns"):
        ringx.ringx_qkv_norm_rope(a["qkv"], 3, 2, a["freqs"], a["rot"], pos=a["pos"])
    with pytest.raises(ValueError, match="contiguous"):
        ringx.ringx_qkv_norm_rope(a["qkv"].transpose(1, 2), 2, 2, a["freqs"], a["rot"], pos=a["pos"])
    with pytest.raises(ringx.RingxError, match="ROPE"):
        forward(a, 2, 2, eps=0.0)
    g = grads_of(9, 1, 10, 2, 2, 64)
    with pytest.raises(ValueError, match="dv: shape"):
        backward(a, g[0], g[1], g[2][:, :1].contiguous())
    with pytest.raises(ValueError, match="without the weight"):
        backward(dict(a, qw=None), *g, dq_weight=torch.empty(64, device="cuda"))


@pytest.mark.parametrize("store,d", [("bf16", 64), ("bf16", 128), ("fp32", 48)])
def test_one_block_together(store, d):
    """Projection -> norm and rotation -> attention with dropout -> gradients -> back to the
    projection, each part against the oracle on what the part before gave."""
    B, N, H, Hkv, p, scale = 2, 150, 4, 2, 0.2, 0.1
    rot = (d // 8 * 2, d // 8 * 2, d // 8 * 2)
    a, x = make(10, B, N, H, Hkv, d, rot, store, pad=64)
    q, k, v = forward(a, H, Hkv)
    rng = state()
    out, lse = ringx.ringx_attn_fwd_drop(q, k, v, p, rng, scale=scale)
    do = torch.randn(out.shape, generator=torch.Generator(device="cuda").manual_seed(1),
                     device="cuda").to(out.dtype)
    grads = ringx.ringx_attn_bwd_drop(q, k, v, out, do, lse, p, rng, scale=scale)
    back = backward(a, *grads)
    check_forward(x, H, Hkv, store, q, k, v)
    y = {"q": to_host_f64(q), "k": to_host_f64(k), "v": to_host_f64(v), "do": to_host_f64(do)}
    ro, rl, z = od.attention_drop(y["q"], y["k"], y["v"], scale, p, SEED)
    b, b_lse = bounds(y, ro, rl, z, scale, store, Hkv)
    ref = dict(zip(("dq", "dk", "dv"), od.attention_drop_bwd(y["q"], y["k"], y["v"], ro, y["do"], rl,
                                                             scale, z)), out=ro)
    got = dict(zip(("dq", "dk", "dv"), grads), out=out)
    for name in ref:
        assert (np.abs(to_host_f64(got[name]) - ref[name]) <= 1.01 * b[name] + 1e-12).all(), name
    assert np.abs(to_host_f64(lse) - rl).max() <= b_lse
    check_backward(x, H, Hkv, store, grads, *back)
