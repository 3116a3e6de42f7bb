"""Plain fp64 CPU oracle for layer norm and the linear layer with its epilogue, forward and backward.

TEST INFRASTRUCTURE ONLY, like the other oracles: numpy, no code of the library.
"""

from __future__ import annotations

import math

import numpy as np

__all__ = ["layer_norm", "layer_norm_bwd", "act", "act_grad", "rows", "unrows", "linear", "linear_bwd"]


def layer_norm(x, w=None, b=None, eps=1e-5):
    """y, mean and 1 / deviation of the rows of x [..., C]."""
    mean = x.mean(-1, keepdims=True)
    r = 1.0 / np.sqrt(((x - mean) ** 2).mean(-1, keepdims=True) + eps)
    y = (x - mean) * r
    y = y if w is None else y * w
    return y if b is None else y + b, mean[..., 0], r[..., 0]


def layer_norm_bwd(x, dy, mean, r, w=None, dres=None):
    """dx, dweight, dbias with the given statistics."""
    mean, r = mean[..., None], r[..., None]
    n = (x - mean) * r
    g = dy if w is None else dy * w
    dx = r * (g - g.mean(-1, keepdims=True) - n * (g * n).mean(-1, keepdims=True))
    axes = tuple(range(x.ndim - 1))
    return dx if dres is None else dx + dres, (dy * n).sum(axes), dy.sum(axes)


_erf = np.vectorize(math.erf, otypes=[np.float64])


def act(z, name):
    if name == "gelu":
        return z * 0.5 * (1.0 + _erf(z / math.sqrt(2.0)))
    if name == "gelu_tanh":
        return 0.5 * z * (1.0 + np.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z ** 3)))
    if name == "silu":
        return z / (1.0 + np.exp(-z))
    return z


def act_grad(z, name):
    if name == "gelu":
        return 0.5 * (1.0 + _erf(z / math.sqrt(2.0))) + z * np.exp(-z * z / 2.0) / math.sqrt(2.0 * math.pi)
    if name == "gelu_tanh":
        u = math.sqrt(2.0 / math.pi)
        t = np.tanh(u * (z + 0.044715 * z ** 3))
        return 0.5 * (1.0 + t) + 0.5 * z * (1.0 - t * t) * u * (1.0 + 3 * 0.044715 * z * z)
    if name == "silu":
        g = 1.0 / (1.0 + np.exp(-z))
        return g * (1.0 + z * (1.0 - g))
    return np.ones_like(z)


def rows(x):
    """x [..., K], or an attention's output [B, H, N, d], as [M, K]."""
    if x.ndim == 4:
        x = x.transpose(0, 2, 1, 3)
        return x.reshape(x.shape[0] * x.shape[1], -1)
    return x.reshape(-1, x.shape[-1])


def unrows(y, like):
    """[M, K] in the layout of `like`."""
    if like.ndim == 4:
        B, H, N, d = like.shape
        return y.reshape(B, N, H, d).transpose(0, 2, 1, 3)
    return y.reshape(like.shape)


def linear(x, w, b=None, name="none", residual=None):
    """y and the activation's input, [M, O]."""
    z = rows(x) @ w.T
    z = z if b is None else z + b
    y = act(z, name)
    return y if residual is None else y + residual.reshape(y.shape), z


def linear_bwd(x, w, dy, pre=None, name="none"):
    """dx in x's layout, dw, dbias."""
    dz = dy.reshape(-1, w.shape[0])
    if name != "none":
        dz = dz * act_grad(pre.reshape(dz.shape), name)
    return unrows(dz @ w, x), dz.T @ rows(x), dz.sum(0)
