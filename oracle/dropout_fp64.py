"""Plain fp64 CPU oracle for attention with dropout on its probabilities.

TEST INFRASTRUCTURE ONLY, like the other oracles: numpy, no code of the library.

    P = softmax(scale q k^T), lse its log-sum-exp; z_ij = m_ij / (1 - T / 256); out = (P z) v;
    dV = (P z)^T dO;  dP = (dO v^T) z;  dS = P (dP - D), D_i = dO_i . out_i;
    dQ = scale dS k;  dK = scale dS^T q.

The mask m is that of Philox4x32 (J. K. Salmon, M. A. Moraes, R. O. Dror, D. E. Shaw, "Parallel
random numbers: as easy as 1, 2, 3", SC'11) with 7 rounds: key = (seed mod 2^32, seed div 2^32),
counter = (2 J + h, query, head, offset mod 2^32) for keys 32 J + 8 m + 4 h + e, whose byte is byte e
of word m; a score is kept iff its byte is at least T = round(256 p).
"""

from __future__ import annotations

import numpy as np

__all__ = ["philox4x32", "threshold", "keep_mask", "head_attention_drop", "head_attention_drop_bwd",
           "attention_drop", "attention_drop_bwd"]

_LOW = np.uint64(0xFFFFFFFF)


def philox4x32(counter, key, rounds=7):
    """Philox4x32: counter (4 arrays), key (2 ints), each 32 bits; the four result words as uint64."""
    c = [np.asarray(x, dtype=np.uint64) for x in counter]
    k = [int(x) for x in key]
    for _ in range(rounds):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> np.uint64(32)) ^ c[1] ^ np.uint64(k[0]), b & _LOW,
             (a >> np.uint64(32)) ^ c[3] ^ np.uint64(k[1]), a & _LOW]
        k = [(k[0] + 0x9E3779B9) % 2 ** 32, (k[1] + 0xBB67AE85) % 2 ** 32]
    return np.broadcast_arrays(*c)


def threshold(p):
    """T = round(256 p) of the rate as the library receives it (fp32)."""
    return int(np.rint(256.0 * float(np.float32(p))))


def keep_mask(seed, offset, head, queries, keys, p):
    """[queries, keys] truth values of one head for integer arrays of places."""
    i, j = np.asarray(queries, np.int64)[:, None], np.asarray(keys, np.int64)[None, :]
    words = philox4x32([(2 * (j // 32) + j // 4 % 2).astype(np.uint64), i.astype(np.uint64),
                        np.uint64(head), np.uint64(int(offset) % 2 ** 32)],
                       [int(seed) % 2 ** 32, int(seed) // 2 ** 32 % 2 ** 32])
    m = j % 32 // 8
    word = np.select([m == 0, m == 1, m == 2], words[:3], words[3])
    return (word >> (8 * (j % 4)).astype(np.uint64)) & np.uint64(255) >= np.uint64(threshold(p))


def head_attention_drop(q, k, v, scale, z):
    """out, lse of one head; z [Nq, Nk]: the mask times its weight."""
    s = scale * (q @ k.T)
    top = s.max(axis=1, keepdims=True)
    e = np.exp(s - top)
    total = e.sum(axis=1, keepdims=True)
    return (e / total * z) @ v, (top + np.log(total))[:, 0]


def head_attention_drop_bwd(q, k, v, out, do, lse, scale, z):
    """dq, dk, dv of one head."""
    P = np.exp(scale * (q @ k.T) - lse[:, None])
    dS = P * ((do @ v.T) * z - (do * out).sum(axis=1, keepdims=True))
    return scale * (dS @ k), scale * (dS.T @ q), (P * z).T @ do


def _weights(q, k, p, rng, q0, key0):
    """z of every head, [B, H, Nq, Nk]."""
    B, H, Nq, _ = q.shape
    Nk = k.shape[2]
    w = 256.0 / (256 - threshold(p))
    return np.stack([keep_mask(rng[0], rng[1], i, q0 + np.arange(Nq), key0 + np.arange(Nk), p) * w
                     for i in range(B * H)]).reshape(B, H, Nq, Nk)


def attention_drop(q, k, v, scale, p, rng, q0=0, key0=0):
    """out [B,H,Nq,d], lse [B,H,Nq] and z for q [B,H,Nq,d], k, v [B,Hkv,Nk,d]; rng = (seed, offset)."""
    B, H = q.shape[:2]
    G = H // k.shape[1]
    z = _weights(q, k, p, rng, q0, key0)
    r = [[head_attention_drop(q[b, h], k[b, h // G], v[b, h // G], scale, z[b, h])
          for h in range(H)] for b in range(B)]
    return (np.stack([np.stack([x[0] for x in y]) for y in r]),
            np.stack([np.stack([x[1] for x in y]) for y in r]), z)


def attention_drop_bwd(q, k, v, out, do, lse, scale, z):
    """dq, and dk, dv summed over the query heads of each group."""
    B, H = q.shape[:2]
    G = H // k.shape[1]
    dq, dk, dv = np.zeros_like(q), np.zeros_like(k), np.zeros_like(v)
    for b in range(B):
        for h in range(H):
            m = h // G
            x = head_attention_drop_bwd(q[b, h], k[b, m], v[b, m], out[b, h], do[b, h], lse[b, h],
                                        scale, z[b, h])
            dq[b, h] = x[0]
            dk[b, m] += x[1]
            dv[b, m] += x[2]
    return dq, dk, dv
