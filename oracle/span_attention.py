"""Attention under spans, oracle side (test infrastructure only), numpy fp64.

Query i of sample j sees the keys lo[j, i] <= k < hi[j, i].  Scores x = scale q.k may be capped, c = cap tanh(x / cap), and get a
bias -slope[head] |i - k|; query head e uses key/value head e / (heads / kv_heads).  An empty span gives a row of zeros, lse = -inf
and no gradient.  Hidden elements are not touched at all, whatever they hold.
"""
import numpy as np


def spans(s, b, causal=True, window=0, documents=None, prefix=None):
    """lo, hi [b, s]; documents, prefix: [s, b] or None."""
    lo, hi = np.zeros((b, s), dtype=np.int64), np.zeros((b, s), dtype=np.int64)
    for j in range(b):
        ids = documents[:, j] if documents is not None else np.zeros(s, dtype=np.int64)
        first = 0
        for end in range(1, s + 1):
            if end < s and ids[end] == ids[first]:
                continue
            for i in range(first, end):
                if ids[first] < 0:
                    continue
                lo[j, i], hi[j, i] = first, end
                if causal:
                    hi[j, i] = i + 1
                    if prefix is not None:
                        hi[j, i] = max(i + 1, first + min(max(int(prefix[first, j]), 0), end - first))
                if window:
                    lo[j, i], hi[j, i] = max(lo[j, i], i - window + 1), min(hi[j, i], i + window)
            first = end
    return lo, hi


def _split(qkv, heads, kv_heads):
    s, b, row = qkv.shape
    x = qkv.reshape(s, b, heads + 2 * kv_heads, -1)
    return x[:, :, :heads], x[:, :, heads:heads + kv_heads], x[:, :, heads + kv_heads:]


def _scores(q, k, i, keys, scale, cap, slope):
    """t and its derivative with respect to q.k, of one query."""
    x = scale * (k @ q)
    d = np.full_like(x, scale)
    if cap:
        th = np.tanh(x / cap)
        x, d = cap * th, d * (1 - th * th)
    return x - slope * np.abs(i - keys), d


def forward(qkv, lo, hi, heads, kv_heads, scale, cap=0.0, slopes=None):
    """Returns ctx [s, b, heads dh], lse [b, heads, s]."""
    q, k, v = _split(qkv, heads, kv_heads)
    s, b, _, dh = q.shape
    ctx, lse = np.zeros((s, b, heads, dh)), np.full((b, heads, s), -np.inf)
    for j in range(b):
        for e in range(heads):
            g = e // (heads // kv_heads)
            slope = 0.0 if slopes is None else slopes[e]
            for i in range(s):
                keys = np.arange(lo[j, i], hi[j, i])
                if keys.size == 0:
                    continue
                t, _ = _scores(q[i, j, e], k[keys, j, g], i, keys, scale, cap, slope)
                m = t.max()
                p = np.exp(t - m)
                lse[j, e, i] = m + np.log(p.sum())
                ctx[i, j, e] = (p / p.sum()) @ v[keys, j, g]
    return ctx.reshape(s, b, -1), lse


def backward(dctx, qkv, lo, hi, heads, kv_heads, scale, cap=0.0, slopes=None):
    """Gradient of qkv."""
    q, k, v = _split(qkv, heads, kv_heads)
    s, b, _, dh = q.shape
    do = dctx.reshape(s, b, heads, dh)
    dq, dk, dv = np.zeros(q.shape), np.zeros(k.shape), np.zeros(v.shape)
    for j in range(b):
        for e in range(heads):
            g = e // (heads // kv_heads)
            slope = 0.0 if slopes is None else slopes[e]
            for i in range(s):
                keys = np.arange(lo[j, i], hi[j, i])
                if keys.size == 0:
                    continue
                t, d = _scores(q[i, j, e], k[keys, j, g], i, keys, scale, cap, slope)
                p = np.exp(t - t.max())
                p /= p.sum()
                dp = v[keys, j, g] @ do[i, j, e]
                dx = p * (dp - p @ dp) * d
                dq[i, j, e] += dx @ k[keys, j, g]
                dk[keys, j, g] += dx[:, None] * q[i, j, e]
                dv[keys, j, g] += p[:, None] * do[i, j, e]
    return np.concatenate((dq, dk, dv), axis=2).reshape(qkv.shape)
