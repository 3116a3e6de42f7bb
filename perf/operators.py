"""Timed cases of two operators around and in the attention: attention with dropout on its
probabilities (forward, and training steps with the backward that recomputes them), and the per-head
norm of queries and keys with their rotation by position, forward and backward.

`run` computes them in plain torch operations, or, where `own` is true, by the library's entry points.
`exact` computes the same in 64 bits, written apart from both.
"""

import math

import torch

own = False

DEVICE = "cuda"
EPS = 1e-6


# ------------------------------------------------------------------------------------------------
# cases


def _attn(name, dtype, B, H, Hkv, Nq, Nk, d, p, bwd):
    return {"name": name, "kind": "attn", "dtype": dtype, "B": B, "H": H, "Hkv": Hkv, "Nq": Nq,
            "Nk": Nk, "d": d, "p": p, "bwd": bwd}


def _rope(name, dtype, B, N, H, Hkv, d, rot, grid, weight, pad, bwd):
    """rot: rotated dims of the position's axes (one, or z, y and x), as "16,24,24"; grid: positions
    are those of a token grid, else consecutive; pad: columns of the projection that are not q, k, v."""
    return {"name": name, "kind": "rope", "dtype": dtype, "B": B, "N": N, "H": H, "Hkv": Hkv, "d": d,
            "rot": rot, "grid": grid, "weight": weight, "pad": pad, "bwd": bwd}


def listed():
    return [
        # a unit test or a toy model: one training step of a few microseconds of work
        _attn("attn_tiny_step", "bf16", 1, 2, 2, 200, 700, 128, 0.1, True),
        # the forward over a batch of short sequences, 6 heads of 128, odd length
        _attn("attn_batch_fwd", "bf16", 4, 6, 6, 1001, 1001, 128, 0.25, False),
        # an fp32 reference training step on 1024 tokens
        _attn("attn_fp32_step", "fp32", 1, 2, 2, 1024, 1024, 64, 0.2, True),
        # the forward over one 16^3 token grid, 16 heads of 64
        _attn("attn_grid16_fwd", "bf16", 1, 16, 16, 4096, 4096, 64, 0.1, False),
        # grouped-query training step at sizes that fit no tile
        _attn("attn_gqa_step", "bf16", 2, 16, 4, 1500, 5003, 64, 0.15, True),
        # one rank's training step of an 8-way ring over a 32^3 token grid, 16 heads of 128
        _attn("attn_ring8_step", "bf16", 1, 16, 16, 4096, 32768, 128, 0.1, True),
        # a single token: latency
        _rope("rope_one_token", "bf16", 1, 1, 16, 16, 128, "128", False, True, 0, False),
        # one rank's 32768 tokens of a 64^3 grid, 16 heads of 128, rotated along z, y and x
        _rope("rope_grid_fwd", "bf16", 1, 32768, 16, 16, 128, "40,44,44", True, True, 0, False),
        # fp32, a head dim and sections that fit no vector, columns of a wider projection
        _rope("rope_fp32_fwd", "fp32", 3, 1531, 3, 3, 100, "30,34,34", True, True, 36, False),
        # backward of a batch of grouped-query heads, part of each head rotated
        _rope("rope_gqa_bwd", "bf16", 2, 4097, 16, 4, 64, "48", False, True, 0, True),
        # backward of the rank's tokens above
        _rope("rope_grid_bwd", "bf16", 1, 32768, 16, 16, 128, "40,44,44", True, True, 0, True),
        # one block's attention, both directions: projection -> norm, rotation -> attention with
        # dropout -> and back, over a 16^3 grid
        {"name": "block_step", "kind": "block", "dtype": "bf16", "B": 1, "N": 4096, "H": 16,
         "Hkv": 16, "d": 64, "rot": "20,22,22", "grid": True, "weight": True, "pad": 0, "p": 0.1},
    ]


def _log(rng, lo, hi):
    """An integer whose logarithm is uniform over [lo, hi]."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _sections(rng, d):
    """Even section sizes that fit d dims."""
    if rng.random() < 0.5:
        return str(d // 2 * 2 if rng.random() < 0.6 else 2 * rng.randint(1, d // 2))
    cut = sorted(rng.randint(1, d // 2) for _ in range(3))
    return ",".join(str(2 * max(1, b - a)) for a, b in zip([0] + cut[:2], cut)) if d >= 12 else "2"


def draw(rng):
    kind = rng.choice(["attn", "attn", "attn", "fp32", "rope", "rope", "rope", "block"])
    Hkv = rng.choice([1, 2, 3, 4, 8, 16])
    H = Hkv * rng.choice([1, 1, 2, 4]) if Hkv <= 4 else Hkv
    B = rng.choice([1, 1, 2, 4])
    p = round(rng.uniform(0.02, 0.5), 3)
    if kind == "attn":
        Nq = _log(rng, 1, 4096)
        Nk = min(32768, max(64, int(Nq * math.exp(rng.uniform(0.0, math.log(8.0))))))
        c = _attn(None, "bf16", 1 if H * Nq > 8192 else B, H, Hkv, Nq, Nk, rng.choice([64, 128]), p,
                  rng.random() < 0.6)
    elif kind == "fp32":
        d = rng.choice([16, 32, 64, 100, 128, rng.randint(1, 128)])
        c = _attn(None, "fp32", 1, min(H, 4), min(Hkv, H, 4) if min(H, 4) % min(Hkv, H, 4) == 0 else 1,
                  _log(rng, 16, 1531), _log(rng, 64, 3001), d, p, rng.random() < 0.5)
    elif kind == "rope":
        dtype = rng.choice(["bf16", "bf16", "fp32"])
        d = rng.choice([64, 128]) if dtype == "bf16" else rng.choice([32, 64, 100, 128,
                                                                      rng.randint(12, 128)])
        rot = _sections(rng, d)
        c = _rope(None, dtype, B, _log(rng, 1, 8192 if B > 1 else 32768), H, Hkv, d, rot,
                  "," in rot, rng.random() < 0.8, rng.choice([0, 0, 64]), rng.random() < 0.5)
    else:
        d = rng.choice([64, 128])
        rot = _sections(rng, d)
        c = {"kind": "block", "dtype": "bf16", "B": 1, "N": _log(rng, 64, 4096), "H": H, "Hkv": Hkv,
             "d": d, "rot": rot, "grid": "," in rot, "weight": rng.random() < 0.8, "pad": 0, "p": p}
    c.pop("name", None)
    return c


# ------------------------------------------------------------------------------------------------
# inputs


def _rot(c):
    return tuple(int(r) for r in c["rot"].split(","))


def _dtype(c):
    return torch.float32 if c["dtype"] == "fp32" else torch.bfloat16


def prepare(case, seed):
    c, dtype = case, _dtype(case)
    gen = torch.Generator(device=DEVICE).manual_seed(int(seed))

    def randn(shape, std, dt):
        return torch.randn(shape, generator=gen, device=DEVICE, dtype=torch.float32).mul_(std).to(dt)

    s = {"case": c}
    if c["kind"] != "rope":
        # the generator's state: seed and step counter
        s["rng"] = torch.randint(0, 1 << 31, (2,), generator=gen, device=DEVICE, dtype=torch.int64)
        s["rng"][0].mul_(0x9E3779B1)
    if c["kind"] == "attn":
        # spreads as in the library's workloads
        std, do_std = ((1.0, 1.0) if c["dtype"] == "fp32" else
                       (0.5, 1.0) if c["d"] == 64 else (2 ** -0.5, 2 ** -0.5))
        B, H, Hkv, d = c["B"], c["H"], c["Hkv"], c["d"]
        s["q"] = randn((B, H, c["Nq"], d), std, dtype)
        s["k"] = randn((B, Hkv, c["Nk"], d), std, dtype)
        s["v"] = randn((B, Hkv, c["Nk"], d), std, dtype)
        if c["bwd"]:
            s["do"] = randn((B, H, c["Nq"], d), do_std, dtype)
        return s
    B, N, H, Hkv, d = c["B"], c["N"], c["H"], c["Hkv"], c["d"]
    rot = _rot(c)
    # the projection's output, whose rows may hold other columns too
    s["qkv"] = randn((B, N, (H + 2 * Hkv) * d + c["pad"]), 1.0, dtype)[:, :, :(H + 2 * Hkv) * d]
    # frequencies of every axis, radians per position
    s["freqs"] = torch.cat([10000.0 ** (-torch.arange(0, r, 2, device=DEVICE, dtype=torch.float64) / r)
                            for r in rot])
    s["pos"] = None
    if c["grid"]:
        # tokens of a 64-wide grid, x fastest, from a rank's first token on
        t = torch.arange(N, device=DEVICE, dtype=torch.int32) + 98304
        s["pos"] = torch.stack([t // 4096, t // 64 % 64, t % 64], 1).contiguous()
    s["qw"] = s["kw"] = None
    if c["weight"]:
        s["qw"] = 1.0 + randn((d,), 0.2, torch.float32)
        s["kw"] = 1.0 + randn((d,), 0.2, torch.float32)
    if c["kind"] == "block":
        s["do"] = randn((B, H, N, d), 1.0, dtype)
    elif c["bwd"]:
        s["dq"] = randn((B, H, N, d), 1.0, torch.float32)
        s["dk"] = randn((B, Hkv, N, d), 1.0, torch.float32)
        s["dv"] = randn((B, Hkv, N, d), 1.0, torch.float32)
    return s


POS0 = 98304   # a rank's first position where positions are consecutive


# ------------------------------------------------------------------------------------------------
# plain forms, in 32 bits


def _mul(c, m):
    """(high, low) 32 bits of the product of c (32 bits in 64) and m; the 64-bit product may wrap into
    the sign, which the masks take off."""
    x = c * m
    return (x >> 32) & 0xFFFFFFFF, x & 0xFFFFFFFF


def _keep(rng, B, H, Nq, Nk, p):
    """[B, H, Nq, Nk] truth values: Philox4x32-7 over (16 keys of a 32-key block, query, head, offset)."""
    nb = (Nk + 31) // 32
    new = dict(device=rng.device, dtype=torch.int64)
    c0 = torch.arange(2 * nb, **new)
    c1 = torch.arange(Nq, **new)[:, None]
    c2 = torch.arange(B * H, **new)[:, None, None]
    c3 = rng[1] & 0xFFFFFFFF
    k0, k1 = rng[0] & 0xFFFFFFFF, (rng[0] >> 32) & 0xFFFFFFFF
    for _ in range(7):
        h0, l0 = _mul(c0, 0xD2511F53)
        h1, l1 = _mul(c2, 0xCD9E8D57)
        c0, c1, c2, c3 = h1 ^ c1 ^ k0, l1, h0 ^ c3 ^ k1, l0
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    words = torch.stack([c0, c1, c2, c3], -1).to(torch.int32)       # [BH, Nq, 2 nb, 4 words]
    x = words.view(torch.uint8).view(B * H, Nq, nb, 2, 4, 4)         # block, half, word, byte
    x = x.transpose(3, 4).reshape(B, H, Nq, 32 * nb)[..., :Nk]       # key 8 word + 4 half + byte
    return x >= int(round(256.0 * p))


def _plain_attn(q, k, v, do, p, rng):
    B, H, Nq, d = q.shape
    Hkv, Nk = k.shape[1], k.shape[2]
    kappa = (256 - int(round(256.0 * p))) / 256.0
    scale = 1.0 / math.sqrt(d)
    fq, fk, fv = q.float().view(B, Hkv, -1, d), k.float(), v.float()
    keep = _keep(rng, B, H, Nq, Nk, p).view(B, Hkv, -1, Nk)
    S = torch.matmul(fq, fk.transpose(2, 3)) * scale
    m = S.amax(-1, keepdim=True)
    P = (S - m).exp_()
    l = P.sum(-1, keepdim=True)
    P = P / l
    lse = (m + l.log()).view(B, H, Nq)
    Z = P * keep / kappa
    o = torch.matmul(Z, fv)
    out = {"out": o.view(B, H, Nq, d).to(q.dtype), "lse": lse}
    if do is not None:
        fdo = do.float().view(B, Hkv, -1, d)
        D = (fdo * o).sum(-1, keepdim=True)
        dS = P * (torch.matmul(fdo, fv.transpose(2, 3)) * keep / kappa - D) * scale
        out["dq"] = torch.matmul(dS, fk).view(B, H, Nq, d)
        out["dk"] = torch.matmul(dS.transpose(2, 3), fq)
        out["dv"] = torch.matmul(Z.transpose(2, 3), fdo)
    return out


def _angles(c, s):
    """cos, sin [N, rotated dims / 2] in 32 bits, the angles in 64."""
    N, rot = c["N"], _rot(c)
    if s["pos"] is None:
        pos = (torch.arange(N, device=DEVICE, dtype=torch.float64) + POS0)[:, None]
    else:
        pos = s["pos"].double()
    axis = torch.repeat_interleave(torch.arange(len(rot), device=DEVICE),
                                   torch.tensor([r // 2 for r in rot], device=DEVICE))
    a = pos[:, axis] * s["freqs"]
    return a.cos().float(), a.sin().float()


def _pairs(c):
    """Dims of the first and the second members of the rotated pairs, and the dims left alone."""
    rot, first, at = _rot(c), [], 0
    for r in rot:
        first += range(at, at + r // 2)
        at += r
    lo = torch.tensor(first, device=DEVICE)
    half = torch.repeat_interleave(torch.tensor([r // 2 for r in rot], device=DEVICE),
                                   torch.tensor([r // 2 for r in rot], device=DEVICE))
    return lo, lo + half


def _turn(y, cos, sin, lo, hi):
    z = y.clone()
    z[..., lo] = y[..., lo] * cos - y[..., hi] * sin
    z[..., hi] = y[..., hi] * cos + y[..., lo] * sin
    return z


def _split(c, x):
    """[B, N, cols] -> q, k, v as [B, heads, N, d]."""
    B, N, H, Hkv, d = c["B"], c["N"], c["H"], c["Hkv"], c["d"]
    x = x.reshape(B, N, H + 2 * Hkv, d).transpose(1, 2)
    return x[:, :H], x[:, H:H + Hkv], x[:, H + Hkv:]


def _plain_rope(c, s):
    q, k, v = _split(c, s["qkv"])
    cos, sin = _angles(c, s)
    lo, hi = _pairs(c)

    def one(x, w):
        x = x.float()
        y = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
        return _turn(y if w is None else y * w, cos, sin, lo, hi).to(s["qkv"].dtype)

    return {"q": one(q, s["qw"]), "k": one(k, s["kw"]), "v": v.contiguous()}


def _plain_rope_bwd(c, s, dq, dk, dv):
    q, k, _ = _split(c, s["qkv"])
    cos, sin = _angles(c, s)
    lo, hi = _pairs(c)
    out = {}

    def one(x, dy, w, name):
        x = x.float()
        r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
        g = _turn(dy, cos, -sin, lo, hi)
        xr = x * r
        if w is not None:
            out[name] = (g * xr).sum((0, 1, 2))
            g = g * w
        return r * (g - xr * (g * xr).mean(-1, keepdim=True))

    dx = torch.cat([one(q, dq, s["qw"], "dq_weight"), one(k, dk, s["kw"], "dk_weight"), dv], 1)
    out["dqkv"] = dx.transpose(1, 2).reshape(c["B"], c["N"], -1).to(s["qkv"].dtype)
    return out


# ------------------------------------------------------------------------------------------------
# one pass


def _own_rope(c, s):
    from paper_2507_16697_amd import ringx
    return ringx.ringx_qkv_norm_rope(s["qkv"], c["H"], c["Hkv"], s["freqs"], _rot(c), pos=s["pos"],
                                     pos0=POS0 if s["pos"] is None else 0, q_weight=s["qw"],
                                     k_weight=s["kw"], eps=EPS)


def _own_rope_bwd(c, s, dq, dk, dv):
    from paper_2507_16697_amd import ringx
    dx, dqw, dkw = ringx.ringx_qkv_norm_rope_bwd(s["qkv"], dq, dk, dv, s["freqs"], _rot(c),
                                                 pos=s["pos"], pos0=POS0 if s["pos"] is None else 0,
                                                 q_weight=s["qw"], k_weight=s["kw"], eps=EPS)
    return {"dqkv": dx} | ({"dq_weight": dqw, "dk_weight": dkw} if c["weight"] else {})


def _own_attn(q, k, v, do, p, rng):
    from paper_2507_16697_amd import ringx
    out, lse = ringx.ringx_attn_fwd_drop(q, k, v, p, rng)
    r = {"out": out, "lse": lse}
    if do is not None:
        r["dq"], r["dk"], r["dv"] = ringx.ringx_attn_bwd_drop(q, k, v, out, do, lse, p, rng)
    return r


def run(state):
    s, c = state, state["case"]
    attn, rope, rope_bwd = ((_own_attn, _own_rope, _own_rope_bwd) if own else
                            (_plain_attn, _plain_rope, _plain_rope_bwd))
    if c["kind"] == "attn":
        r = attn(s["q"], s["k"], s["v"], s.get("do"), c["p"], s["rng"])
        if c["bwd"]:
            # to the inputs' type, as the backward of the projections takes them
            r.update((x, r[x].to(s["q"].dtype)) for x in ("dq", "dk", "dv"))
        return r
    if c["kind"] == "rope":
        if c["bwd"]:
            return rope_bwd(c, s, s["dq"], s["dk"], s["dv"])
        r = rope(c, s)
        return r if isinstance(r, dict) else dict(zip("qkv", r))
    r = rope(c, s)
    q, k, v = (r["q"], r["k"], r["v"]) if isinstance(r, dict) else r
    a = attn(q, k, v, s["do"], c["p"], s["rng"])
    g = rope_bwd(c, s, a["dq"], a["dk"], a["dv"])
    # a training program steps its weights in their own type
    return {"out": a["out"], "dqkv": g["dqkv"]} | {
        x: g[x].to(s["qkv"].dtype) for x in ("dq_weight", "dk_weight") if x in g}


# ------------------------------------------------------------------------------------------------
# what a pass cannot do without


def work(case):
    c = case
    es = 4 if c["dtype"] == "fp32" else 2
    B, H, Hkv, d = c["B"], c["H"], c["Hkv"], c["d"]
    if c["kind"] == "attn":
        nq, nkv, rows = B * H * c["Nq"] * d, B * Hkv * c["Nk"] * d, B * H * c["Nq"]
        pairs = 2 * B * H * c["Nq"] * c["Nk"] * d          # one contraction
        n = es * (2 * nq + 2 * nkv) + 4 * rows              # q, k, v, out, lse
        if not c["bwd"]:
            return {"bytes": n, "flops": 2 * pairs}
        return {"bytes": n + es * (2 * nq + 2 * nkv), "flops": 6 * pairs}    # and dO, dq, dk, dv
    cols, rows = (H + 2 * Hkv) * d, B * c["N"]
    if c["kind"] == "rope":
        if c["bwd"]:
            return {"bytes": rows * cols * (2 * es + 4), "flops": 12 * rows * cols}
        return {"bytes": rows * cols * 2 * es, "flops": 7 * rows * cols}
    pairs = 2 * B * H * c["N"] ** 2 * d
    return {"bytes": es * (2 * rows * cols + 2 * rows * H * d), "flops": 6 * pairs + 19 * rows * cols}


# ------------------------------------------------------------------------------------------------
# the same results in 64 bits


def _philox_bytes(seed, offset, head, Nq, Nk):
    """[Nq, Nk] mask bytes of one head, by 16-bit partial products."""
    nb = (Nk + 31) // 32

    def wide(a, m):
        al, ah, ml, mh = a & 0xFFFF, a >> 16, m & 0xFFFF, m >> 16
        mid = ah * ml + ((al * ml) >> 16)
        mid2 = al * mh + (mid & 0xFFFF)
        return ah * mh + (mid >> 16) + (mid2 >> 16), ((mid2 & 0xFFFF) << 16) | ((al * ml) & 0xFFFF)

    def full(x):
        return torch.as_tensor(x, device=DEVICE, dtype=torch.int64).expand(Nq, 2 * nb)

    ctr = [full(torch.arange(2 * nb, device=DEVICE)), full(torch.arange(Nq, device=DEVICE)[:, None]),
           full(head), full(offset % 2 ** 32)]
    key = [seed % 2 ** 32, (seed >> 32) % 2 ** 32]
    for i in range(7):
        a, b = wide(ctr[0], 0xD2511F53), wide(ctr[2], 0xCD9E8D57)
        ctr = [b[0] ^ ctr[1] ^ key[0], b[1], a[0] ^ ctr[3] ^ key[1], a[1]]
        key = [(key[0] + 0x9E3779B9) % 2 ** 32, (key[1] + 0xBB67AE85) % 2 ** 32]
    j = torch.arange(Nk, device=DEVICE)
    col = 2 * (j // 32) + j // 4 % 2
    word = torch.stack(ctr)[j % 32 // 8, :, col].t()
    return (word >> (8 * (j % 4))) & 255


def _exact_attn(q, k, v, do, p, rng):
    B, H, Nq, d = q.shape
    Hkv, Nk = k.shape[1], k.shape[2]
    seed, offset = (int(x) for x in rng.tolist())
    T = int(round(256.0 * p))
    new = dict(dtype=torch.float64, device=q.device)
    r = {"out": torch.empty((B, H, Nq, d), **new), "lse": torch.empty((B, H, Nq), **new)}
    if do is not None:
        r.update(dq=torch.empty((B, H, Nq, d), **new), dk=torch.zeros((B, Hkv, Nk, d), **new),
                 dv=torch.zeros((B, Hkv, Nk, d), **new))
    for b in range(B):
        for h in range(H):
            m = h // (H // Hkv)
            qq, kk, vv = q[b, h].double(), k[b, m].double(), v[b, m].double()
            z = (_philox_bytes(seed, offset, b * H + h, Nq, Nk) >= T).double() * (256.0 / (256 - T))
            s = qq @ kk.t() / math.sqrt(d)
            lse = torch.logsumexp(s, 1)
            P = torch.exp(s - lse[:, None])
            o = (P * z) @ vv
            r["out"][b, h], r["lse"][b, h] = o, lse
            if do is not None:
                dd = do[b, h].double()
                dp = (dd @ vv.t()) * z
                ds = P * (dp - (P * dp).sum(1, keepdim=True)) / math.sqrt(d)
                r["dq"][b, h] = ds @ kk
                r["dk"][b, m] += ds.t() @ qq
                r["dv"][b, m] += (P * z).t() @ dd
    return r


def _exact_rope(c, s, grads=None):
    """q, k, v, or with the gradients of these those of the projection and the weights."""
    B, N, H, Hkv, d = c["B"], c["N"], c["H"], c["Hkv"], c["d"]
    x = s["qkv"].double().reshape(B, N, H + 2 * Hkv, d)
    # the rotation as a complex factor of every pair
    at, f0, parts = 0, 0, []
    for a, r in enumerate(_rot(c)):
        pos = (torch.arange(N, device=DEVICE).double() + POS0 if s["pos"] is None
               else s["pos"][:, a].double())
        ang = torch.outer(pos, s["freqs"][f0:f0 + r // 2])
        parts.append((at, r // 2, torch.complex(ang.cos(), ang.sin())[:, None]))
        at, f0 = at + r, f0 + r // 2

    def turn(y, back=False):
        y = y.clone()
        for a, n, z in parts:
            u = torch.complex(y[..., a:a + n], y[..., a + n:a + 2 * n]) * (z.conj() if back else z)
            y[..., a:a + n], y[..., a + n:a + 2 * n] = u.real, u.imag
        return y

    one = torch.ones(d, device=DEVICE, dtype=torch.float64)
    w = torch.cat([(one if s["qw"] is None else s["qw"].double()).expand(H, d),
                   (one if s["kw"] is None else s["kw"].double()).expand(Hkv, d)])
    y = x[:, :, :H + Hkv]
    r = 1.0 / torch.sqrt((y * y).mean(-1, keepdim=True) + EPS)
    n = y * r
    if grads is None:
        z = turn(n * w).permute(0, 2, 1, 3)
        return {"q": z[:, :H].contiguous(), "k": z[:, H:].contiguous(),
                "v": x[:, :, H + Hkv:].permute(0, 2, 1, 3).contiguous()}
    g = [t.double().permute(0, 2, 1, 3) for t in grads]
    t = turn(torch.cat(g[:2], 2), back=True)
    dw = (t * n).sum((0, 1))
    t = t * w
    dx = r * (t - n * (t * n).mean(-1, keepdim=True))
    res = {"dqkv": torch.cat([dx, g[2]], 2).reshape(B, N, -1)}
    if c["weight"]:
        res.update(dq_weight=dw[:H].sum(0), dk_weight=dw[H:].sum(0))
    return res


def exact(case, seed):
    c = case
    s = prepare(c, seed)
    if c["kind"] == "attn":
        return _exact_attn(s["q"], s["k"], s["v"], s.get("do"), c["p"], s["rng"])
    if c["kind"] == "rope":
        return _exact_rope(c, s, (s["dq"], s["dk"], s["dv"]) if c["bwd"] else None)
    f = _exact_rope(c, s)
    a = _exact_attn(f["q"], f["k"], f["v"], s["do"], c["p"], s["rng"])
    g = _exact_rope(c, s, (a["dq"], a["dk"], a["dv"]))
    return {"out": a["out"], "dqkv": g["dqkv"]} | {
        x: g[x] for x in ("dq_weight", "dk_weight") if x in g}
