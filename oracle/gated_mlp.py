"""Gated feed-forward block, oracle side (test infrastructure only), numpy fp64.

z = u w with columns [gate | up], g = f(z_gate + b_gate) (z_up + b_up); with dg = dy w2^T: dz_gate = dg f'(a) c, dz_up = dg f(a).
"""
import math

import numpy as np

_erf = np.vectorize(math.erf)


def _sigmoid(a):
    return 1 / (1 + np.exp(-a))


def act(kind, a):
    """f(a) and f'(a)."""
    if kind == "silu":
        s = _sigmoid(a)
        return a * s, s + a * s * (1 - s)
    if kind == "gelu_erf":
        cdf = 0.5 * (1 + _erf(a / math.sqrt(2)))
        return a * cdf, cdf + a * np.exp(-a * a / 2) / math.sqrt(2 * math.pi)
    if kind == "gelu_tanh":
        c = math.sqrt(2 / math.pi)
        t = np.tanh(c * (a + 0.044715 * a ** 3))
        return 0.5 * a * (1 + t), 0.5 * (1 + t) + 0.5 * a * (1 - t * t) * c * (1 + 3 * 0.044715 * a * a)
    if kind == "sigmoid":
        s = _sigmoid(a)
        return s, s * (1 - s)
    return np.maximum(a, 0), (a > 0).astype(a.dtype)   # relu


def forward(kind, u, w, bias=None):
    z = u @ w
    a, c = np.split(z + (0 if bias is None else bias), 2, axis=-1)
    return z, act(kind, a)[0] * c


def backward(kind, dy, w2, z, bias=None):
    a, c = np.split(z + (0 if bias is None else bias), 2, axis=-1)
    f, d = act(kind, a)
    dg = dy @ w2.T
    return np.concatenate((dg * d * c, dg * f), axis=-1)
