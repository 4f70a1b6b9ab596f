"""Rotary positions, oracle side (test infrastructure only): pairs of elements as complex numbers, numpy fp64.

A head's first `rot` elements are rot / 2 pairs, (i, i + rot/2) or neighbours; pair i of a token at position p is multiplied by
amplitude * exp(2 pi sqrt(-1) p turns[i]).  Backward: by the conjugate.
"""
import numpy as np


def turns(rot, base=10000.0, scaling="plain", factor=1.0, trained=1.0, slow=0.0, fast=1.0):
    """Turns per position of every pair."""
    i = np.arange(rot // 2)
    if scaling == "base":
        base = base * factor ** (rot / (rot - 2))
    f = base ** (-2.0 * i / rot) / (2 * np.pi)
    if scaling == "linear":
        f = f / factor
    if scaling == "ramp":
        g = np.clip((trained * f - slow) / (fast - slow), 0.0, 1.0)
        f = f * (g + (1 - g) / factor)
    return f


def _pairs(x, rot, neighbours):
    r = x[..., :rot]
    return r[..., 0::2] + 1j * r[..., 1::2] if neighbours else r[..., :rot // 2] + 1j * r[..., rot // 2:]


def rotate(x, positions, f, heads, kv_heads, rot, neighbours, amplitude=1.0, back=False):
    """x [s, b, (heads + 2 kv_heads) dh]; positions [s, b] or None (the token index); returns the turned rows."""
    s, b, row = x.shape
    dh = row // (heads + 2 * kv_heads)
    if positions is None:
        positions = np.repeat(np.arange(s)[:, None], b, axis=1)
    turn = positions[..., None].astype(np.float64) * f
    z = amplitude * np.exp((-2j if back else 2j) * np.pi * (turn - np.round(turn)))
    out = x.reshape(s, b, heads + 2 * kv_heads, dh).copy()
    y = _pairs(out[:, :, :heads + kv_heads], rot, neighbours) * z[:, :, None]
    if neighbours:
        out[:, :, :heads + kv_heads, 0:rot:2] = y.real
        out[:, :, :heads + kv_heads, 1:rot:2] = y.imag
    else:
        out[:, :, :heads + kv_heads, :rot // 2] = y.real
        out[:, :, :heads + kv_heads, rot // 2:rot] = y.imag
    return out.reshape(s, b, row)
