"""Plain fp64 CPU oracle for the per-head RMS norm of queries and keys with their rotation by position.

TEST INFRASTRUCTURE ONLY, like the other oracles: numpy, no code of the library.

For a row x of d dims (one token, one head): r = (mean x^2 + eps)^(-1/2), y = x r w; section a of the
rotated dims turns its pairs (o + i, o + n + i), i < n, by position_a f_{a, i}.  The backward turns the
gradient back (g) and gives dw = sum g x r and dx = r (g w - x r mean(g w x r)).
"""

from __future__ import annotations

import numpy as np

__all__ = ["turn", "qkv_norm_rope", "qkv_norm_rope_bwd"]


def turn(y, pos, freqs, rot, back=False):
    """y [..., N, d] turned by the angles of pos [..., N, axes]."""
    z = np.array(y, dtype=np.float64)
    o = f = 0
    for a, dims in enumerate(rot):
        n = dims // 2
        t = pos[..., a, None].astype(np.float64) * freqs[f:f + n]
        c, s = np.cos(t), -np.sin(t) if back else np.sin(t)
        lo, hi = y[..., o:o + n], y[..., o + n:o + 2 * n]
        z[..., o:o + n] = lo * c - hi * s
        z[..., o + n:o + 2 * n] = hi * c + lo * s
        o, f = o + 2 * n, f + n
    return z


def _heads(qkv, H, Hkv):
    """[B, heads, N, d] of a packed projection."""
    B, N, cols = qkv.shape
    d = cols // (H + 2 * Hkv)
    x = qkv.reshape(B, N, H + 2 * Hkv, d).transpose(0, 2, 1, 3)
    return x[:, :H], x[:, H:H + Hkv], x[:, H + Hkv:]


def _positions(pos, pos0, N):
    if pos is None:
        return (np.arange(N) + pos0)[:, None]
    return pos[:, None] if pos.ndim == 3 else pos     # [B, 1, N, axes] or [N, axes]


def qkv_norm_rope(qkv, H, Hkv, freqs, rot, pos=None, pos0=0, qw=None, kw=None, eps=1e-6):
    q, k, v = _heads(qkv, H, Hkv)
    p = _positions(pos, pos0, qkv.shape[1])

    def one(x, w):
        y = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
        return turn(y if w is None else y * w, p, freqs, rot)

    return one(q, qw), one(k, kw), v


def qkv_norm_rope_bwd(qkv, dq, dk, dv, freqs, rot, pos=None, pos0=0, qw=None, kw=None, eps=1e-6):
    """dqkv [B, N, cols], dq_weight, dk_weight."""
    q, k, _ = _heads(qkv, dq.shape[1], dk.shape[1])
    p = _positions(pos, pos0, qkv.shape[1])

    def one(x, dy, w):
        r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
        g = turn(dy, p, freqs, rot, back=True)
        dw = (g * x * r).sum((0, 1, 2))
        g = g if w is None else g * w
        return r * (g - x * r * (g * x * r).mean(-1, keepdims=True)), dw

    dxq, dqw = one(q, dq, qw)
    dxk, dkw = one(k, dk, kw)
    dx = np.concatenate([dxq, dxk, dv], 1).transpose(0, 2, 1, 3)
    return dx.reshape(qkv.shape[0], qkv.shape[1], -1), dqw, dkw
