"""Attention with dropout on the GPU against the fp64 oracle: forward, backward, ring steps, both
types, grouped heads, lengths from one token on, places on the mask's axes, graphs and streams.

Bounds are those of rounding: P, dS and the stored output to bf16 (2^-8 of the value each), fp32
arithmetic elsewhere, carried through each contraction with absolute values."""

import math

import numpy as np
import pytest
import torch

from oracle import dropout_fp64 as od
from paper_2507_16697_amd import inputs, ring, ringx

from parity_util import to_device, to_host_f64

pytestmark = pytest.mark.gpu

SEED = (0x1234_5678_9ABC_DEF1, 0x3_0000_0007)     # seed; offset beyond 32 bits, taken mod 2^32


def state(seed=SEED):
    return torch.tensor(seed, dtype=torch.int64, device="cuda")


def case(seed, B, H, Hkv, Nq, Nk, d, store):
    std = 1.0 if store == "fp32" else (0.5 if d == 64 else 2 ** -0.5)
    a = inputs.make_iid(B, H, Nq, 1, d, seed=seed, std=std, store=store)
    b = inputs.make_iid(B, Hkv, 1, Nk, d, seed=seed + 1000, std=std, store=store, with_do=False)
    t = {"q": a["q"], "do": a["do"], "k": b["k"], "v": b["v"]}
    return ({n: to_device(x, store) for n, x in t.items()},
            {n: inputs.to_f64(x, store) for n, x in t.items()})


def bounds(x, out, lse, z, scale, store, dkv_heads):
    """Element-wise error bounds of out, dq, dk, dv, and one of lse."""
    B, H = x["q"].shape[:2]
    G = H // dkv_heads
    rep = lambda t: np.repeat(t, G, axis=1)   # noqa: E731
    T = lambda t: np.swapaxes(t, -1, -2)      # noqa: E731
    q, k, v, do = x["q"], rep(x["k"]), rep(x["v"]), x["do"]
    d, Nk, Nq = q.shape[-1], k.shape[2], q.shape[2]
    e = 2.0 ** -24
    u = 2.0 ** -8 if store == "bf16" else 0.0
    # a score: d products and sums, the scale, the exponent's subtraction; the exponential 2^-21
    size = scale * (np.abs(q) @ T(np.abs(k)))
    ds = float(size.max()) * (d + 8) * e + 4 * e * float(np.abs(lse).max()) + 2.0 ** -21
    P = np.exp(scale * (q @ T(k)) - lse[..., None])
    Z = P * z
    rel = u + 2 * ds + (Nk + 32) * e           # a probability's rounding, the row sum's, the product's
    b_out = rel * (Z @ np.abs(v)) + (u + 4 * e) * np.abs(out)
    dP = (do @ T(v)) * z
    D = (do * out).sum(-1, keepdims=True)
    b_D = (np.abs(do) * b_out).sum(-1, keepdims=True) + (d + 4) * e * (np.abs(do) * np.abs(out)).sum(
        -1, keepdims=True)
    dS = P * (dP - D)
    E = (u + 2 * ds + 8 * e) * np.abs(dS) + P * (
        b_D + (d + 8) * e * ((np.abs(do) @ T(np.abs(v))) * z + np.abs(D)))
    s = np.abs(dS)
    b_dq = scale * (E @ np.abs(k) + (Nk + 8) * e * (s @ np.abs(k)))
    b_dk = scale * (T(E) @ np.abs(q) + (G * Nq + 8) * e * (T(s) @ np.abs(q)))
    b_dv = (u + 2 * ds + (G * Nq + 8) * e) * (T(Z) @ np.abs(do))
    fold = lambda t: t.reshape(B, dkv_heads, G, *t.shape[2:]).sum(2)   # noqa: E731
    b_lse = ds + (Nk + 32) * e + 8 * e * float(np.abs(lse).max())
    return {"out": b_out, "dq": b_dq, "dk": fold(b_dk), "dv": fold(b_dv)}, b_lse


def check(x, got, p, rng, scale, store, q0=0, key0=0):
    """got: out, lse (, dq, dk, dv) device tensors."""
    ro, rl, z = od.attention_drop(x["q"], x["k"], x["v"], scale, p, rng, q0, key0)
    b, b_lse = bounds(x, ro, rl, z, scale, store, x["k"].shape[1])
    ref = {"out": ro}
    if "dq" in got:
        ref["dq"], ref["dk"], ref["dv"] = od.attention_drop_bwd(x["q"], x["k"], x["v"], ro, x["do"],
                                                                rl, scale, z)
    assert float(np.max(np.abs(to_host_f64(got["lse"]) - rl))) <= b_lse
    for name, r in ref.items():
        err = np.abs(to_host_f64(got[name]) - r)
        over = err - b[name] * 1.0001 - 1e-12
        assert np.isfinite(err).all() and over.max() <= 0, (name, float(err.max()), float(over.max()))


def both(g, p, rng, scale, **kw):
    out, lse = ringx.ringx_attn_fwd_drop(g["q"], g["k"], g["v"], p, rng, scale=scale, **kw)
    dq, dk, dv = ringx.ringx_attn_bwd_drop(g["q"], g["k"], g["v"], out, g["do"], lse, p, rng,
                                           scale=scale, **kw)
    return {"out": out, "lse": lse, "dq": dq, "dk": dk, "dv": dv}


def f32_scale(d):
    return float(np.float32(1 / math.sqrt(d)))


# sizes that take each form of a launch: one token, less than a tile, tiles that end inside, key
# streams, half-size workgroups, whole workgroups
@pytest.mark.parametrize("store,B,H,Hkv,Nq,Nk,d,p", [
    ("bf16", 1, 1, 1, 1, 1, 128, 0.5), ("bf16", 1, 1, 1, 1, 1, 64, 0.5),
    ("bf16", 2, 2, 1, 1, 333, 64, 0.1), ("bf16", 1, 2, 2, 33, 31, 128, 0.3),
    ("bf16", 1, 2, 2, 200, 700, 128, 0.1), ("bf16", 1, 4, 2, 257, 513, 64, 0.25),
    ("bf16", 2, 6, 2, 300, 1000, 128, 0.15), ("bf16", 1, 3, 3, 64, 2049, 64, 0.9),
    ("bf16", 1, 36, 36, 513, 190, 64, 0.1), ("bf16", 1, 36, 36, 513, 190, 128, 0.1),
    ("bf16", 1, 70, 70, 1025, 130, 64, 0.2), ("bf16", 1, 70, 35, 1025, 130, 128, 0.2),
    ("bf16", 1, 130, 26, 270, 515, 64, 0.2),
    ("bf16", 1, 130, 130, 520, 70, 64, 0.2), ("bf16", 1, 8, 4, 300, 4400, 64, 0.2),
    ("bf16", 1, 1, 1, 100, 100, 64, 0.0), ("bf16", 1, 1, 1, 100, 100, 128, 0.0),
    ("fp32", 1, 1, 1, 1, 1, 1, 0.5), ("fp32", 1, 2, 1, 17, 47, 3, 0.2),
    ("fp32", 2, 4, 2, 130, 333, 24, 0.1), ("fp32", 1, 3, 3, 257, 301, 100, 0.3),
    ("fp32", 1, 2, 2, 100, 515, 128, 0.1), ("fp32", 1, 6, 1, 64, 64, 64, 0.0)])
def test_forward_and_backward(store, B, H, Hkv, Nq, Nk, d, p):
    print(f"dropout {store} B={B} H={H}/{Hkv} Nq={Nq} Nk={Nk} d={d} p={p}", flush=True)
    g, x = case(Nq + 7 * Nk + d, B, H, Hkv, Nq, Nk, d, store)
    got = both(g, p, state(), f32_scale(d))
    check(x, got, p, SEED, f32_scale(d), store)


# few heads: sweeps in parts that are summed afterwards, on both sides, on one, with shared heads; the
# last part ends inside a tile
@pytest.mark.parametrize("B,H,Hkv,Nq,Nk,d", [
    (1, 2, 2, 1111, 1333, 64), (1, 4, 1, 517, 2100, 128), (1, 1, 1, 300, 2100, 64), (1, 1, 1, 1, 1030, 128),
    (2, 3, 1, 2051, 77, 128), (1, 6, 2, 1030, 333, 64)])
def test_split_sweeps(B, H, Hkv, Nq, Nk, d):
    print(f"split B={B} H={H}/{Hkv} Nq={Nq} Nk={Nk} d={d}", flush=True)
    args = (B, H, Hkv, Nq, Nk, d, ringx.RINGX_BF16)
    need = ringx.ringx_bwd_drop_workspace_bytes(*args)
    assert need > ringx.ringx_bwd_workspace_bytes(B, H, Nq, Nk, d, 1, ringx.RINGX_BF16)
    g, x = case(Nq + Nk, B, H, Hkv, Nq, Nk, d, "bf16")
    p, scale, kw = 0.2, f32_scale(d), dict(q0=77, key0=64)
    got = both(g, p, state(), scale, **kw)
    check(x, got, p, SEED, scale, "bf16", **kw)
    # what a workspace held before does not matter, nothing behind it is written, and a sum onto given
    # gradients is the sum
    ws = torch.full((need + 256,), 255, dtype=torch.uint8, device="cuda")
    fwd_need = ringx.ringx_fwd_drop_workspace_bytes(*args)
    if fwd_need:
        fws = torch.full((fwd_need + 256,), 255, dtype=torch.uint8, device="cuda")
        out, lse = ringx.ringx_attn_fwd_drop(g["q"], g["k"], g["v"], p, state(), scale=scale,
                                             workspace=fws[:fwd_need], **kw)
        assert torch.equal(out, got["out"]) and torch.equal(lse, got["lse"])
        assert bool((fws[fwd_need:] == 255).all())
    acc = {n: torch.randn_like(got[n]) for n in ("dk", "dv")}
    old = {n: t.clone() for n, t in acc.items()}
    dq, _, _ = ringx.ringx_attn_bwd_drop(g["q"], g["k"], g["v"], got["out"], g["do"], got["lse"], p, state(),
                                         scale=scale, dk=acc["dk"], dv=acc["dv"], accumulate_dkv=True,
                                         workspace=ws[:need], **kw)
    assert torch.equal(dq, got["dq"]) and bool((ws[need:] == 255).all())
    assert all(torch.equal(acc[n], old[n] + got[n]) for n in acc)


@pytest.mark.parametrize("store,d", [("bf16", 128), ("bf16", 64), ("fp32", 40)])
def test_places_on_the_mask_axes(store, d):
    """Parts of the queries and of the keys with their places draw the whole call's mask; places far out
    too."""
    g, x = case(5, 1, 2, 2, 120, 256, d, store)
    scale, p = f32_scale(d), 0.3
    for q0, key0 in ((0, 0), (4_000_000_000, (1 << 36) - 320)):
        got = both(g, p, state(), scale, q0=q0, key0=key0)
        check(x, got, p, SEED, scale, store, q0, key0)
    whole = ringx.ringx_attn_fwd_drop(g["q"], g["k"], g["v"], p, state(), scale=scale)[0]
    part = ringx.ringx_attn_fwd_drop(g["q"][:, :, 50:].contiguous(), g["k"], g["v"], p, state(),
                                     scale=scale, q0=50)[0]
    b, _ = bounds(x, *od.attention_drop(x["q"], x["k"], x["v"], scale, p, SEED), scale, store, 2)
    err = np.abs(to_host_f64(part) - to_host_f64(whole)[:, :, 50:])
    assert (err <= 2 * b["out"][:, :, 50:]).all()


def test_no_rate_is_plain_attention():
    # 700 keys: too few for parts of their own, so to the bit
    g, x = case(6, 1, 2, 2, 300, 700, 128, "bf16")
    o, l = ringx.ringx_attn_fwd_drop(g["q"], g["k"], g["v"], 0.0, state())
    ro, rl = ringx.ringx_attn_fwd(g["q"], g["k"], g["v"], 1)
    assert torch.equal(o, ro) and torch.equal(l, rl)


@pytest.mark.parametrize("store,d", [("bf16", 64), ("bf16", 128), ("fp32", 64)])
def test_repeats_and_accumulates(store, d):
    g, _ = case(8, 1, 4, 2, 300, 700, d, store)
    a, b = both(g, 0.2, state(), f32_scale(d)), both(g, 0.2, state(), f32_scale(d))
    assert all(torch.equal(a[n], b[n]) for n in a)
    base = torch.randn_like(a["dk"])
    dk, dv = base.clone(), base.clone()
    ringx.ringx_attn_bwd_drop(g["q"], g["k"], g["v"], a["out"], g["do"], a["lse"], 0.2, state(),
                              scale=f32_scale(d), dk=dk, dv=dv, accumulate_dkv=True)
    assert torch.equal(dk, base + a["dk"]) and torch.equal(dv, base + a["dv"])
    other = both(g, 0.2, state((SEED[0], SEED[1] + 1)), f32_scale(d))
    assert torch.equal(other["lse"], a["lse"]) and not torch.equal(other["out"], a["out"])


# Every mask that a score can have, exactly: with all scores equal and V the identity on 32 keys, an
# output is m_ij / (kappa Nk).
@pytest.mark.parametrize("store", ["bf16", "fp32"])
def test_forward_mask_bit_by_bit(store):
    H, Nq, d = 3, 70, 64
    dt = torch.bfloat16 if store == "bf16" else torch.float32
    q = torch.zeros((1, H, Nq, d), device="cuda", dtype=dt)
    k = torch.zeros((1, H, d, d), device="cuda", dtype=dt)
    v = torch.eye(d, device="cuda", dtype=dt).expand(1, H, d, d).contiguous()
    for p in (1 / 256, 0.3, 255 / 256):
        out, _ = ringx.ringx_attn_fwd_drop(q, k, v, p, state(), q0=9, key0=96)
        for h in range(H):
            m = od.keep_mask(*SEED, h, 9 + np.arange(Nq), 96 + np.arange(d), p)
            assert np.array_equal(out[0, h].float().cpu().numpy() > 0, m)


@pytest.mark.parametrize("store,d,lengths", [("bf16", 128, (256, 256, 192)), ("bf16", 64, (96, 32, 300)),
                                             ("fp32", 36, (64, 160, 50)), ("bf16", 64, (33, 100, 7))])
def test_ring_steps(store, d, lengths):
    """The ring against the oracle with every chunk at its place; chunks of whole blocks give the mask
    of one call."""
    g, x = case(9, 1, 2, 2, 130, sum(lengths), d, store)
    p, scale = 0.2, f32_scale(d)
    at = np.cumsum((0,) + lengths)
    kc = [g["k"][:, :, a:b].contiguous() for a, b in zip(at, at[1:])]
    vc = [g["v"][:, :, a:b].contiguous() for a, b in zip(at, at[1:])]
    out, lse = ring.ring_forward(g["q"], kc, vc, scale=scale, dropout=(p, state()), q0=77)
    dq, dk, dv = ring.ring_backward(g["q"], kc, vc, out, g["do"], lse, scale=scale,
                                    dropout=(p, state()), q0=77)
    places = np.concatenate([s + np.arange(n) for s, n in zip(ring.mask_places(lengths), lengths)])
    w = 256 / (256 - od.threshold(p))
    z = np.stack([od.keep_mask(*SEED, h, 77 + np.arange(130), places, p) * w for h in range(2)])[None]
    res = [od.head_attention_drop(x["q"][0, h], x["k"][0, h], x["v"][0, h], scale, z[0, h])
           for h in range(2)]
    ro, rl = np.stack([r[0] for r in res])[None], np.stack([r[1] for r in res])[None]
    ref = dict(zip(("dq", "dk", "dv"), od.attention_drop_bwd(x["q"], x["k"], x["v"], ro, x["do"], rl,
                                                             scale, z)))
    ref["out"] = ro
    b, b_lse = bounds(x, ro, rl, z, scale, store, 2)
    got = {"out": out, "dq": dq, "dk": torch.cat(dk, 2), "dv": torch.cat(dv, 2)}
    for name in ref:
        assert (np.abs(to_host_f64(got[name]) - ref[name]) <= 1.01 * b[name] + 1e-12).all(), name
    assert np.abs(to_host_f64(lse) - rl).max() <= 2 * b_lse
    if all(n % 32 == 0 for n in lengths[:-1]):
        one = both(g, p, state(), scale, q0=77)
        assert (np.abs(to_host_f64(one["out"]) - to_host_f64(out)) <= 2.01 * b["out"]).all()


def test_fp32_gradient_is_a_difference():
    """The forward's outputs, not only the formula, have the backward's gradient."""
    g, x = case(10, 1, 1, 1, 40, 70, 16, "fp32")
    p, scale, h = 0.3, 0.25, 2.0 ** -6
    got = both(g, p, state(), scale)
    ro, rl, z = od.attention_drop(x["q"], x["k"], x["v"], scale, p, SEED)
    b, _ = bounds(x, ro, rl, z, scale, "fp32", 1)
    for name, grad in (("q", "dq"), ("k", "dk"), ("v", "dv")):
        dirn = np.random.default_rng(3).standard_normal(x[name].shape).astype(np.float32)
        dirn = np.round(dirn * 16) / 16                     # x + h dirn is exact enough: fp32 of both

        def loss_gpu(t):
            y = dict(g)
            y[name] = g[name] + t * torch.from_numpy(dirn.astype(np.float32)).cuda()
            o = ringx.ringx_attn_fwd_drop(y["q"], y["k"], y["v"], p, state(), scale=scale)[0]
            return float((to_host_f64(o) * x["do"]).sum())

        def loss_ref(t):
            y = dict(x)
            y[name] = x[name] + t * dirn
            return float((od.attention_drop(y["q"], y["k"], y["v"], scale, p, SEED)[0] * x["do"]).sum())

        num = (loss_gpu(h) - loss_gpu(-h)) / (2 * h)
        num_ref = (loss_ref(h) - loss_ref(-h)) / (2 * h)
        exact = float((od.attention_drop_bwd(x["q"], x["k"], x["v"], ro, x["do"], rl, scale, z)[
            ("q", "k", "v").index(name)] * dirn).sum())
        truncation = abs(num_ref - exact)
        # the outputs' rounding, and the rounding of the moved input (2^-24 of about 4, times gradient)
        noise = 2 * float((np.abs(x["do"]) * b["out"]).sum()) / h
        noise += 2.0 ** -21 / h * float(np.abs(to_host_f64(got[grad])).sum())
        mine = float((to_host_f64(got[grad]) * dirn).sum())
        assert abs(num - mine) <= truncation + noise + float((b[grad] * np.abs(dirn)).sum())


def test_infinite_key_features_stay_where_they_are():
    """A key masked by features that make its score -inf adds nothing, dropped or not."""
    g, x = case(11, 1, 2, 2, 100, 200, 64, "bf16")
    g["q"][..., 0] = 1.0
    g["k"][..., 0] = 0.0
    g["k"][:, :, 150:, 0] = -float("inf")
    out, lse = ringx.ringx_attn_fwd_drop(g["q"], g["k"], g["v"], 0.2, state())
    ref, rl = ringx.ringx_attn_fwd_drop(g["q"], g["k"][:, :, :150].contiguous(),
                                        g["v"][:, :, :150].contiguous(), 0.2, state())
    assert torch.isfinite(out).all() and torch.allclose(lse, rl, atol=1e-5, rtol=0)
    # the same probabilities, summed in other tiles: a rounding of P and one of out each, of sums
    # whose weights add up to at most 256 / (256 - T)
    most = 256 / (256 - od.threshold(0.2)) * float(g["v"].abs().max())
    assert float((out.float() - ref.float()).abs().max()) <= 4 * 2 ** -8 * most


@pytest.mark.parametrize("d", [64, 128])
def test_parts_of_the_keys_without_a_finite_score(d):
    """Few queries: the keys go to workgroups in parts, most of which hold scores of -inf alone; the
    same for the chunks of a ring after the first."""
    Nk, some = 2048, 200
    g, _ = case(14, 1, 2, 2, 70, Nk, d, "bf16")
    assert ringx.ringx_fwd_drop_workspace_bytes(1, 2, 2, 70, Nk, d, ringx.RINGX_BF16) > 0
    g["q"][..., 0] = 1.0
    g["k"][..., 0] = 0.0
    g["k"][:, :, some:, 0] = -float("inf")
    out, lse = ringx.ringx_attn_fwd_drop(g["q"], g["k"], g["v"], 0.2, state())
    ref, rl = ringx.ringx_attn_fwd_drop(g["q"], g["k"][:, :, :some].contiguous(),
                                        g["v"][:, :, :some].contiguous(), 0.2, state())
    most = 256 / (256 - od.threshold(0.2)) * float(g["v"].abs().max())   # as above
    assert torch.allclose(lse, rl, atol=1e-5, rtol=0)
    assert float((out.float() - ref.float()).abs().max()) <= 4 * 2 ** -8 * most
    dq = ringx.ringx_attn_bwd_drop(g["q"], g["k"], g["v"], out, g["do"], lse, 0.2, state())[0]
    assert torch.isfinite(dq[..., 1:]).all()
    acc = torch.empty((1, 2, 70, d), device="cuda")
    al = torch.empty((1, 2, 70), device="cuda")
    for i, lo in enumerate((0, 1024)):
        ringx.ringx_attn_fwd_step_drop(g["q"], g["k"][:, :, lo:lo + 1024].contiguous(),
                                       g["v"][:, :, lo:lo + 1024].contiguous(), acc, al, i == 0, 0.2,
                                       state(), lo)
    assert torch.allclose(al, rl, atol=1e-5, rtol=0)
    assert float((acc - ref.float()).abs().max()) <= 4 * 2 ** -8 * most


def test_graph_draws_a_new_mask_when_the_state_moves():
    g, x = case(12, 1, 2, 2, 300, 520, 64, "bf16")
    p, scale, rng = 0.25, f32_scale(64), state()
    res = both(g, p, rng, scale)                      # the buffers, and a warm start
    ws = torch.empty(ringx.ringx_bwd_drop_workspace_bytes(1, 2, 2, 300, 520, 64, ringx.RINGX_BF16),
                     dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        ringx.ringx_attn_fwd_drop(g["q"], g["k"], g["v"], p, rng, scale=scale, out=res["out"],
                                  lse=res["lse"])
        ringx.ringx_attn_bwd_drop(g["q"], g["k"], g["v"], res["out"], g["do"], res["lse"], p, rng,
                                  scale=scale, dq=res["dq"], dk=res["dk"], dv=res["dv"],
                                  workspace=ws)
    torch.cuda.synchronize()
    for step in range(3):
        rng.copy_(torch.tensor((SEED[0], step), dtype=torch.int64))
        graph.replay()
        torch.cuda.synchronize()
        eager = both(g, p, state((SEED[0], step)), scale)
        torch.cuda.synchronize()
        assert all(torch.equal(res[n], eager[n]) for n in res), step


def test_two_streams_at_once():
    cases = [case(20 + i, 1, 2, 2, 300, 700, d, "bf16")[0] for i, d in enumerate((64, 128))]
    want = [both(g, 0.2, state(), 0.1) for g in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    rng = state()
    torch.cuda.synchronize()
    got = []
    for g, s in zip(cases, streams):
        with torch.cuda.stream(s):
            got.append(both(g, 0.2, rng, 0.1))
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        assert all(torch.equal(a[n], b[n]) for n in a)


def test_binding_refusals():
    g, _ = case(13, 1, 2, 2, 40, 64, 64, "bf16")
    q, k, v = g["q"], g["k"], g["v"]
    for bad in (torch.zeros(3, dtype=torch.int64, device="cuda"), torch.zeros(2, device="cuda")):
        with pytest.raises((ValueError, TypeError), match="rng"):
            ringx.ringx_attn_fwd_drop(q, k, v, 0.1, bad)
    with pytest.raises(ringx.RingxError, match="DROPOUT"):
        ringx.ringx_attn_fwd_drop(q, k, v, 1.0, state())
    with pytest.raises(ringx.RingxError, match="DROPOUT"):
        ringx.ringx_attn_fwd_drop(q, k, v, 0.1, state(), key0=8)
    with pytest.raises(ValueError, match="v: shape"):
        ringx.ringx_attn_fwd_drop(q, k, v[:, :, 1:].contiguous(), 0.1, state())
    with pytest.raises(ValueError, match="contiguous"):
        ringx.ringx_attn_fwd_drop(q.transpose(1, 2), k, v, 0.1, state())
