"""Timed cases of the operators on both sides of the attention in a transformer block: layer norm, and
the matrix product of tokens and weights with bias, activation and residual in its epilogue, forward and
backward, one by one and together as the block's norm and MLP.

`run` computes them in plain torch operations, or, where `own` is true, by the library's entry points.
`exact` computes the same in 64 bits, written apart from both.
"""

import math

import torch

own = False

DEVICE = "cuda"
EPS = 1e-5


# ------------------------------------------------------------------------------------------------
# cases


def _ln(name, dtype, M, C, affine, pad, res, way):
    """M rows of C; affine: weight and bias; pad: columns of the rows that are not normed; res: the
    backward adds the gradient of the residual path; way: fwd, bwd, or step (both)."""
    return {"name": name, "kind": "ln", "dtype": dtype, "M": M, "C": C, "affine": affine, "pad": pad,
            "res": res, "way": way}


def _lin(name, dtype, B, N, K, O, heads, act, bias, res, pre, pad, way):
    """B N rows of K features to O; heads: the rows lie as an attention's output [B, heads, N, K / heads]
    does (0: row by row, pad columns apart); pre: the forward keeps what the backward needs of the
    activation's input; way: fwd, bwd, or step (both)."""
    return {"name": name, "kind": "lin", "dtype": dtype, "B": B, "N": N, "K": K, "O": O,
            "heads": heads, "act": act, "bias": bias, "res": res, "pre": pre, "pad": pad, "way": way}


def _mlp(name, dtype, M, C, F, act):
    return {"name": name, "kind": "mlp", "dtype": dtype, "M": M, "C": C, "F": F, "act": act}


def listed():
    return [
        # a single token's norm: latency
        _ln("ln_one_token", "bf16", 1, 2048, True, 0, False, "fwd"),
        # one rank's 32768 tokens of a 64^3 grid, 16 heads of 128 wide
        _ln("ln_grid_fwd", "bf16", 32768, 2048, True, 0, False, "fwd"),
        # an fp32 reference step over rows of a wider tensor, a width that fits no tile
        _ln("ln_fp32_step", "fp32", 4593, 300, True, 36, False, "step"),
        # backward in a pre-norm block of a batch of odd sequences: the residual's gradient joins in
        _ln("ln_batch_bwd", "bf16", 8194, 960, True, 0, True, "bwd"),
        # the same over the rank's tokens above
        _ln("ln_grid_bwd", "bf16", 32768, 2048, True, 0, True, "bwd"),
        # a single token through the first product of an MLP: latency and the weights' bandwidth
        _lin("lin_one_token", "bf16", 1, 1, 2048, 8192, 0, "gelu", True, False, False, 0, "fwd"),
        # the patch embedding of 17^3 patches of 5^3 cells with 3 components: rows of odd length
        _lin("lin_patch_fwd", "bf16", 1, 4913, 375, 960, 0, "none", True, False, False, 0, "fwd"),
        # the output projection of an attention with 16 heads of 64, with the residual, and back
        _lin("lin_heads_step", "bf16", 2, 4097, 1024, 1024, 16, "none", True, True, False, 0, "step"),
        # the packed projection of the rank's tokens to queries, keys and values
        _lin("lin_qkv_fwd", "bf16", 1, 32768, 2048, 6144, 0, "none", True, False, False, 0, "fwd"),
        # an fp32 reference step of an MLP's first product
        _lin("lin_fp32_step", "fp32", 1, 1531, 192, 577, 0, "gelu", True, False, True, 0, "step"),
        # backward of an MLP's first product at a batch of odd sequences
        _lin("lin_gelu_bwd", "bf16", 2, 4097, 960, 3840, 0, "gelu", True, False, True, 0, "bwd"),
        # norm and MLP of a pre-norm block, both directions, half of the rank's tokens
        _mlp("mlp_step", "bf16", 16384, 2048, 8192, "gelu"),
    ]


def _log(rng, lo, hi):
    """An integer whose logarithm is uniform over [lo, hi]."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _width(rng, lo, hi):
    """A width: mostly whole multiples of 8, as models have them, else any."""
    n = _log(rng, lo, hi)
    return n if rng.random() < 0.25 else max(8, n // 8 * 8)


def draw(rng):
    kind = rng.choice(["ln", "ln", "lin", "lin", "lin", "lin", "mlp"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "fp32"])
    way = rng.choice(["fwd", "bwd", "step"])
    act = rng.choice(["none", "gelu", "gelu", "gelu_tanh", "silu"])
    if kind == "ln":
        C = _width(rng, 16, 16384)
        M = _log(rng, 1, max(1, min(32768, 67108864 // C)))
        pad = rng.choice([0, 0, 8 if C % 8 == 0 or dtype == "fp32" else 5])
        c = _ln(None, dtype, M, C, rng.random() < 0.8, pad, rng.random() < 0.5, way)
    elif kind == "lin":
        heads = rng.choice([0, 0, 0, 2, 3, 8, 16])
        K = heads * rng.choice([64, 128]) if heads else _width(rng, 16, 8192)
        O = _width(rng, 16, 8192)
        most = 1.5e11 if dtype == "bf16" else 1e10
        N = _log(rng, 1, max(1, min(32768, int(most / (K * O)))))
        B = 2 if N > 1 and rng.random() < 0.3 else 1
        c = _lin(None, dtype, B, max(1, N // B), K, O, heads, act, rng.random() < 0.8,
                 way != "bwd" and act == "none" and rng.random() < 0.5, way != "fwd" or rng.random() < 0.4,
                 0 if heads else rng.choice([0, 0, 16]), way)
    else:
        C = 8 * _log(rng, 4, 256)
        F = C * rng.choice([2, 4])
        M = _log(rng, 64, min(16384, int((5e10 if dtype == "bf16" else 4e9) / (C * F))))
        c = _mlp(None, dtype, M, C, F, act if act != "none" else "gelu")
    c.pop("name", None)
    return c


# ------------------------------------------------------------------------------------------------
# inputs


def _dtype(c):
    return torch.float32 if c["dtype"] == "fp32" else torch.bfloat16


def prepare(case, seed):
    c, dtype = case, _dtype(case)
    gen = torch.Generator(device=DEVICE).manual_seed(int(seed))

    def randn(shape, std, dt=dtype, mean=0.0):
        return torch.randn(shape, generator=gen, device=DEVICE).mul_(std).add_(mean).to(dt)

    def stream(M, C, pad=0):
        # a block's running sum: channels of different means and spreads
        x = torch.randn((M, C + pad), generator=gen, device=DEVICE)
        x.mul_(torch.rand(C + pad, generator=gen, device=DEVICE).mul_(3.0).exp_().mul_(0.3))
        x.add_(torch.randn(C + pad, generator=gen, device=DEVICE).mul_(0.5))
        return x.to(dtype)[:, :C]

    f32 = torch.float32
    s = {"case": c}
    if c["kind"] == "ln":
        M, C = c["M"], c["C"]
        s["x"] = stream(M, C, c["pad"])
        s["w"] = randn((C,), 0.2, f32, 1.0) if c["affine"] else None
        s["b"] = randn((C,), 0.2, f32) if c["affine"] else None
        if c["way"] != "fwd":
            s["dy"] = randn((M, C), 1.0)
            s["dres"] = randn((M, C), 1.0) if c["res"] else None
        if c["way"] == "bwd":
            # what the forward kept: mean and 1 / deviation of every row
            x = s["x"].double()
            mean = x.mean(1)
            r = torch.rsqrt((x - mean[:, None]).square_().mean(1) + EPS)
            s["stats"] = torch.stack([mean, r]).float()
        return s
    if c["kind"] == "lin":
        B, N, K, O = c["B"], c["N"], c["K"], c["O"]
        if c["heads"]:
            s["x"] = randn((B, c["heads"], N, K // c["heads"]), 1.0)
        else:
            s["x"] = randn((B, N, K + c["pad"]), 1.0)[:, :, :K]
        s["w"] = randn((O, K), K ** -0.5)
        s["b"] = randn((O,), 0.3, f32) if c["bias"] else None
        s["res"] = randn((B, N, O), 1.0) if c["res"] else None
        if c["way"] != "fwd":
            s["dy"] = randn((B, N, O), 1.0)
        if c["way"] == "bwd":
            # what the forward kept: the activation's input
            s["pre"] = None
            if c["act"] != "none":
                z = torch.matmul(_rows(c, s["x"]).float(), s["w"].float().t())
                s["pre"] = (z if s["b"] is None else z + s["b"]).view(B, N, O).to(dtype)
        return s
    M, C, F = c["M"], c["C"], c["F"]
    s["x"] = stream(M, C)
    s["w"], s["b"] = randn((C,), 0.2, f32, 1.0), randn((C,), 0.2, f32)
    s["w1"], s["b1"] = randn((F, C), C ** -0.5), randn((F,), 0.1, f32)
    s["w2"], s["b2"] = randn((C, F), F ** -0.5), randn((C,), 0.1, f32)
    s["dy"] = randn((M, C), 1.0)
    return s


def _rows(c, x):
    """x as [B N, K]."""
    if c["heads"]:
        x = x.transpose(1, 2)
    return x.reshape(c["B"] * c["N"], c["K"])


def _narrow(c):
    """Whether the bias's gradient is stepped in the inputs' type: it goes through an activation's input
    that the step itself has rounded to it."""
    return c["way"] == "step" and c["act"] != "none" and c["pre"]


# ------------------------------------------------------------------------------------------------
# plain forms, in 32 bits


def _act(z, act):
    if act == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return 0.5 * z * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z * z * z)))
    if act == "silu":
        return z / (1.0 + torch.exp(-z))
    return z


def _act_grad(z, act):
    if act == "gelu":
        return (0.5 * (1.0 + torch.erf(z * math.sqrt(0.5)))
                + z * torch.exp(-0.5 * z * z) * (1.0 / math.sqrt(2.0 * math.pi)))
    if act == "gelu_tanh":
        u = math.sqrt(2.0 / math.pi)
        t = torch.tanh(u * (z + 0.044715 * z * z * z))
        return 0.5 * (1.0 + t) + 0.5 * z * (1.0 - t * t) * u * (1.0 + 3 * 0.044715 * z * z)
    if act == "silu":
        g = 1.0 / (1.0 + torch.exp(-z))
        return g * (1.0 + z * (1.0 - g))
    return torch.ones_like(z)


def _plain_ln(x, w, b):
    """y in 32 bits, and the rows' mean and 1 / deviation."""
    x = x.float()
    mean = x.mean(1, keepdim=True)
    xc = x - mean
    r = torch.rsqrt((xc * xc).mean(1, keepdim=True) + EPS)
    y = xc * r
    if w is not None:
        y = y * w + b
    return y, torch.cat([mean, r], 1).t()


def _plain_ln_bwd(x, dy, stats, w, dres):
    dy = dy.float()
    n = (x.float() - stats[0][:, None]) * stats[1][:, None]
    r = {}
    g = dy
    if w is not None:
        r["dweight"], r["dbias"] = (dy * n).sum(0), dy.sum(0)
        g = dy * w
    dx = stats[1][:, None] * (g - g.mean(1, keepdim=True) - n * (g * n).mean(1, keepdim=True))
    r["dx"] = dx if dres is None else dx + dres.float()
    return r


def _plain_lin(x, w, b, act, res):
    """y and the activation's input, in 32 bits."""
    z = torch.matmul(x.float(), w.float().t())
    if b is not None:
        z = z + b
    y = _act(z, act)
    return (y if res is None else y + res.float()), z


def _plain_lin_bwd(x, w, dy, pre, act, bias):
    dz = dy.float()
    if act != "none":
        dz = dz * _act_grad(pre.float(), act)
    r = {"dx": torch.matmul(dz, w.float()), "dw": torch.matmul(dz.t(), x.float())}
    if bias:
        r["dbias"] = dz.sum(0)
    return r


def _run_plain(c, s):
    dtype = _dtype(c)
    if c["kind"] == "ln":
        out, stats = {}, s.get("stats")
        if c["way"] != "bwd":
            y, stats = _plain_ln(s["x"], s["w"], s["b"])
            out["y"] = y.to(dtype)
        if c["way"] != "fwd":
            g = _plain_ln_bwd(s["x"], s["dy"], stats, s["w"], s["dres"])
            g["dx"] = g["dx"].to(dtype)
            out.update(g)
        return out
    if c["kind"] == "lin":
        B, N, K, O = c["B"], c["N"], c["K"], c["O"]
        x, act = _rows(c, s["x"]), c["act"]
        out, pre = {}, s.get("pre")
        if c["way"] != "bwd":
            y, pre = _plain_lin(x, s["w"], s["b"], act, None if s["res"] is None else s["res"].view(-1, O))
            out["y"] = y.to(dtype).view(B, N, O)
            if c["pre"] and act != "none":
                out["pre"] = pre.to(dtype).view(B, N, O)
                pre = out["pre"]      # the backward's input is what was kept
        if c["way"] != "fwd":
            g = _plain_lin_bwd(x, s["w"], s["dy"].view(-1, O),
                               None if pre is None else pre.view(-1, O), act, c["bias"])
            dx = g["dx"].to(dtype)
            g["dx"] = (dx.view(B, N, c["heads"], -1).transpose(1, 2).contiguous() if c["heads"]
                       else dx.view(B, N, K))
            if act != "none":
                g["dw"] = g["dw"].to(dtype)
            if c["bias"] and _narrow(c):
                g["dbias"] = g["dbias"].to(dtype)
            out.update(g)
        return out
    a, stats = _plain_ln(s["x"], s["w"], s["b"])
    h, z = _plain_lin(a, s["w1"], s["b1"], c["act"], None)
    y, _ = _plain_lin(h, s["w2"], s["b2"], "none", s["x"])
    g2 = _plain_lin_bwd(h, s["w2"], s["dy"], None, "none", True)
    g1 = _plain_lin_bwd(a, s["w1"], g2["dx"], z, c["act"], True)
    g = _plain_ln_bwd(s["x"], g1["dx"], stats, s["w"], s["dy"])
    return _mlp_out(dtype, y, g["dx"], g["dweight"], g["dbias"], g1["dw"], g1["dbias"], g2["dw"],
                    g2["dbias"])


def _mlp_out(dtype, *ts):
    """A step's results in the type in which the program keeps its weights."""
    names = ("y", "dx", "dweight", "dbias", "dw1", "db1", "dw2", "db2")
    return {n: t if t.dtype is dtype else t.to(dtype) for n, t in zip(names, ts)}


# ------------------------------------------------------------------------------------------------
# the library's calls


def _run_own(c, s):
    from paper_2507_16697_amd import ringx
    dtype = _dtype(c)
    if c["kind"] == "ln":
        out, stats = {}, s.get("stats")
        if c["way"] != "bwd":
            out["y"], stats = ringx.ringx_layer_norm(s["x"], s["w"], s["b"], eps=EPS,
                                                     need_stats=c["way"] == "step")
        if c["way"] != "fwd":
            dx, dw, db = ringx.ringx_layer_norm_bwd(s["x"], s["dy"], stats, s["w"], s["b"],
                                                    dres=s["dres"])
            if dw is not None:
                out["dweight"], out["dbias"] = dw, db
            out["dx"] = dx
        return out
    if c["kind"] == "lin":
        out, pre, act = {}, s.get("pre"), c["act"]
        if c["way"] != "bwd":
            keep = c["pre"] and act != "none"
            out["y"], pre = ringx.ringx_linear(s["x"], s["w"], s["b"], act=act, residual=s["res"],
                                               need_pre=keep)
            if keep:
                out["pre"] = pre
        if c["way"] != "fwd":
            dx, dw, db = ringx.ringx_linear_bwd(s["x"], s["w"], s["dy"], pre=pre, act=act, bias=s["b"],
                                                dw_dtype=torch.float32 if act == "none" else dtype)
            out["dx"], out["dw"] = dx, dw
            if db is not None:
                out["dbias"] = db.to(dtype) if _narrow(c) else db
        return out
    a, stats = ringx.ringx_layer_norm(s["x"], s["w"], s["b"], eps=EPS)
    h, z = ringx.ringx_linear(a, s["w1"], s["b1"], act=c["act"], need_pre=True)
    y, _ = ringx.ringx_linear(h, s["w2"], s["b2"], residual=s["x"])
    dh, dw2, db2 = ringx.ringx_linear_bwd(h, s["w2"], s["dy"], bias=s["b2"], dw_dtype=dtype)
    da, dw1, db1 = ringx.ringx_linear_bwd(a, s["w1"], dh, pre=z, act=c["act"], bias=s["b1"],
                                          dx_dtype=torch.float32, dw_dtype=dtype)
    dx, dw, db = ringx.ringx_layer_norm_bwd(s["x"], da, stats, s["w"], s["b"], dres=s["dy"])
    return _mlp_out(dtype, y, dx, dw, db, dw1, db1, dw2, db2)


# ------------------------------------------------------------------------------------------------
# one pass


def run(state):
    return _run_own(state["case"], state) if own else _run_plain(state["case"], state)


# ------------------------------------------------------------------------------------------------
# what a pass cannot do without


def work(case):
    c = case
    es = 4 if c["dtype"] == "fp32" else 2
    if c["kind"] == "ln":
        n, vec = c["M"] * c["C"], 8 * c["C"] if c["affine"] else 0
        nbytes = flops = 0
        if c["way"] != "bwd":
            nbytes, flops = 2 * es * n + vec, 7 * n
        if c["way"] != "fwd":
            # x (once for both directions), dy, the residual's gradient; dx, and the weights' gradients
            nbytes += es * n * (2 + (c["way"] == "bwd") + c["res"]) + vec
            nbytes += 8 * c["M"] + vec // 2 if c["way"] == "bwd" else 0
            flops += 12 * n
        return {"bytes": nbytes, "flops": flops}
    if c["kind"] == "lin":
        M, K, O = c["B"] * c["N"], c["K"], c["O"]
        kept = c["pre"] and c["act"] != "none"
        nbytes, flops = es * (M * K + K * O), 0
        if c["way"] != "bwd":
            nbytes += es * M * O * (1 + c["res"] + kept) + 4 * O * c["bias"]
            flops += 2 * M * K * O
        if c["way"] != "fwd":
            # dy, what was kept; dx, dw, dbias
            nbytes += es * M * O * (1 + (c["way"] == "bwd" and kept)) + es * M * K + 4 * O * c["bias"]
            nbytes += (4 if c["act"] == "none" else es) * K * O
            flops += 4 * M * K * O
        return {"bytes": nbytes, "flops": flops}
    M, C, F = c["M"], c["C"], c["F"]
    # x, dy, y, dx; the weights and their gradients.  What lies between is the step's own.
    return {"bytes": es * (4 * M * C + 4 * C * F) + 4 * (3 * C + F) + es * (3 * C + F),
            "flops": 12 * M * C * F + 19 * M * C}


# ------------------------------------------------------------------------------------------------
# the same results in 64 bits


def _phi(z, act):
    """The activation and its derivative."""
    if act == "gelu":
        p = torch.special.ndtr(z)
        return z * p, p + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if act == "gelu_tanh":
        a = math.sqrt(8 / math.pi)
        g = torch.sigmoid(a * (z + 0.044715 * z ** 3))      # (1 + tanh u) / 2 = sigmoid(2 u)
        return z * g, g + z * g * (1 - g) * a * (1 + 0.134145 * z ** 2)
    if act == "silu":
        g = torch.sigmoid(z)
        return z * g, g + z * g * (1 - g)
    return z, torch.ones_like(z)


def _exact_norm(x, w, b):
    var, mean = torch.var_mean(x, 1, unbiased=False, keepdim=True)
    n = (x - mean) / torch.sqrt(var + EPS)
    y = n if w is None else torch.addcmul(b.double(), n, w.double())
    return y, n, 1 / torch.sqrt(var + EPS)


def _exact_norm_bwd(n, r, dy, w):
    g = dy if w is None else dy * w.double()
    C = n.shape[1]
    dx = r * (g - g.sum(1, keepdim=True) / C - n * ((g * n).sum(1, keepdim=True) / C))
    return dx, torch.einsum("mc,mc->c", dy, n), dy.sum(0)


def exact(case, seed):
    c = case
    s = prepare(c, seed)
    d = {k: t.double() for k, t in s.items() if isinstance(t, torch.Tensor)}
    if c["kind"] == "ln":
        y, n, r = _exact_norm(d["x"], s["w"], s["b"])
        out = {"y": y} if c["way"] != "bwd" else {}
        if c["way"] != "fwd":
            if c["way"] == "bwd":
                # with the statistics as they were kept
                r = d["stats"][1][:, None]
                n = (d["x"] - d["stats"][0][:, None]) * r
            dx, dw, db = _exact_norm_bwd(n, r, d["dy"], s["w"])
            if c["affine"]:
                out.update(dweight=dw, dbias=db)
            out["dx"] = dx + d["dres"] if c["res"] else dx
        return out
    if c["kind"] == "lin":
        B, N, K, O = c["B"], c["N"], c["K"], c["O"]
        x = (d["x"].permute(0, 2, 1, 3) if c["heads"] else d["x"]).reshape(B * N, K)
        out, pre = {}, d.get("pre")
        if c["way"] != "bwd":
            z = x @ d["w"].t()
            if c["bias"]:
                z += d["b"]
            y = _phi(z, c["act"])[0]
            if c["res"]:
                y = y + d["res"].reshape(-1, O)
            out["y"] = y.view(B, N, O)
            if c["pre"] and c["act"] != "none":
                out["pre"] = z.view(B, N, O)
                pre = z.to(_dtype(c)).double()
        if c["way"] != "fwd":
            dz = d["dy"].reshape(-1, O)
            if c["act"] != "none":
                dz = dz * _phi(pre.reshape(-1, O), c["act"])[1]
            dx = dz @ d["w"]
            out["dx"] = (dx.view(B, N, c["heads"], -1).permute(0, 2, 1, 3) if c["heads"]
                         else dx.view(B, N, K)).contiguous()
            out["dw"] = dz.t() @ x
            if c["bias"]:
                out["dbias"] = dz.sum(0)
        return out
    a, n, r = _exact_norm(d["x"], s["w"], s["b"])
    h, slope = _phi(a @ d["w1"].t() + d["b1"], c["act"])
    y = h @ d["w2"].t() + d["b2"] + d["x"]
    dz = (d["dy"] @ d["w2"]) * slope
    dx, dw, db = _exact_norm_bwd(n, r, dz @ d["w1"], s["w"])
    return {"y": y, "dx": dx + d["dy"], "dweight": dw, "dbias": db, "dw1": dz.t() @ a,
            "db1": dz.sum(0), "dw2": d["dy"].t() @ h, "db2": d["dy"].sum(0)}
