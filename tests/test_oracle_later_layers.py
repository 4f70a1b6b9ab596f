"""Pins of the oracles of rotary positions, attention under spans and the gated feed-forward block: differences, closed forms, and independent derivations."""
import numpy as np
import pytest
import torch

from oracle import gpt_layer as L
from oracle import gated_mlp as G, rotary, span_attention as A


@pytest.mark.parametrize("neighbours", [False, True])
def test_rotation_by_hand(neighbours):
    """One pair at position 3 with a twelfth of a turn per position: a quarter turn, (x, y) -> amplitude (-y, x)."""
    x = np.arange(24.0).reshape(1, 1, 24)   # one Q, K and V head of 8; rot 8: four pairs
    got = rotary.rotate(x, np.array([[3]]), np.full(4, 1 / 12), 1, 1, 8, neighbours, amplitude=2.0)[0, 0]
    for h in (0, 8):
        a, b = (x[0, 0, h:h + 8:2], x[0, 0, h + 1:h + 8:2]) if neighbours else (x[0, 0, h:h + 4], x[0, 0, h + 4:h + 8])
        ga, gb = (got[h:h + 8:2], got[h + 1:h + 8:2]) if neighbours else (got[h:h + 4], got[h + 4:h + 8])
        assert np.allclose(ga, -2 * b) and np.allclose(gb, 2 * a)
    assert np.array_equal(got[16:], x[0, 0, 16:])


@pytest.mark.parametrize("neighbours", [False, True])
def test_rotation_gradient_and_relative_positions(neighbours):
    rng = np.random.default_rng(1)
    x, dy = rng.normal(size=(5, 2, 4 * 16)), rng.normal(size=(5, 2, 4 * 16))
    f = rotary.turns(8)
    turn = lambda v, p=None, **kw: rotary.rotate(v, p, f, 2, 1, 8, neighbours, 1.3, **kw)  # noqa: E731
    dx = turn(dy, back=True)
    d = rng.normal(size=x.shape)
    assert np.isclose(((turn(x + 1e-6 * d) - turn(x - 1e-6 * d)) * dy).sum() / 2e-6, (dx * d).sum(), rtol=1e-7)
    # products of turned heads depend on the difference of their positions only
    p = rng.integers(0, 1000, size=(5, 2))
    q, k = (turn(x, p + shift)[..., h:h + 16] for h, shift in ((0, 7), (32, 7)))
    q0, k0 = (turn(x, p)[..., h:h + 16] for h in (0, 32))
    assert np.allclose((q * k[::-1]).sum(-1), (q0 * k0[::-1]).sum(-1))


def test_frequencies():
    f = rotary.turns(64)
    assert np.isclose(f[0], 1 / (2 * np.pi)) and np.isclose(f[31], 10000 ** (-62 / 64) / (2 * np.pi))
    assert np.allclose(rotary.turns(64, scaling="linear", factor=4.0), f / 4)
    # the base form keeps the fastest pair and slows the slowest one by the factor
    g = rotary.turns(64, scaling="base", factor=4.0)
    assert np.isclose(g[0], f[0]) and np.isclose(g[-1], f[-1] / 4)
    r = rotary.turns(64, scaling="ramp", factor=4.0, trained=2048, slow=1.0, fast=32.0)
    fast, slow = 2048 * f >= 32, 2048 * f <= 1
    assert fast.any() and slow.any() and np.allclose(r[fast], f[fast]) and np.allclose(r[slow], f[slow] / 4)
    between = ~fast & ~slow
    assert between.any() and ((r < f) & (r > f / 4))[between].all()


def test_spans_by_hand():
    ids = np.array([[5], [5], [5], [-1], [7], [7], [5]])
    lo, hi = A.spans(7, 1, True, 0, ids)
    assert lo[0].tolist() == [0, 0, 0, 0, 4, 4, 6] and hi[0].tolist() == [1, 2, 3, 0, 5, 6, 7]
    lo, hi = A.spans(7, 1, False, 2, ids)
    assert lo[0].tolist() == [0, 0, 1, 0, 4, 4, 6] and hi[0].tolist() == [2, 3, 3, 0, 6, 6, 7]
    lo, hi = A.spans(7, 1, True, 0, ids, np.array([[2], [9], [9], [9], [9], [0], [-3]]))
    assert hi[0].tolist() == [2, 2, 3, 0, 6, 6, 7]


def test_plain_causal_is_the_layers_attention():
    rng = np.random.default_rng(2)
    s, b, heads, dh = 9, 2, 3, 8
    qkv, dctx = rng.normal(size=(s, b, 3 * heads * dh)), rng.normal(size=(s, b, heads * dh))
    cfg = L.LayerConfig(h=heads * dh, a=heads, t=1, s=s, b=b, causal=True)
    ctx, probs, lse = L.attention_core(qkv, cfg)
    lo, hi = A.spans(s, b)
    got, glse = A.forward(qkv, lo, hi, heads, heads, dh ** -0.5)
    assert np.allclose(got, ctx) and np.allclose(glse, lse)
    assert np.allclose(A.backward(dctx, qkv, lo, hi, heads, heads, dh ** -0.5), L.attention_core_backward(dctx, qkv, probs, cfg))


@pytest.mark.parametrize("cap,bias", [(0.0, False), (2.0, False), (0.0, True), (1.5, True)])
def test_against_differentiated_torch(cap, bias):
    """The same scores as a dense tensor with a mask, gradients by differentiation, shared heads, empty rows."""
    rng = np.random.default_rng(3)
    s, b, heads, kv, dh = 11, 2, 4, 2, 8
    qkv, dctx = rng.normal(size=(s, b, (heads + 2 * kv) * dh)), rng.normal(size=(s, b, heads * dh))
    ids = np.stack([[0] * 4 + [1] * 5 + [-1] * 2, [3] * 11], axis=1)
    slopes = np.array([0.5, 0.25, 0.1, 0.0]) if bias else None
    lo, hi = A.spans(s, b, True, 0, ids)
    ctx, lse = A.forward(qkv, lo, hi, heads, kv, 0.4, cap, slopes)
    x = torch.tensor(qkv, requires_grad=True)
    y = x.view(s, b, heads + 2 * kv, dh)
    q, k, v = y[:, :, :heads], y[:, :, heads:heads + kv].repeat_interleave(2, 2), y[:, :, heads + kv:].repeat_interleave(2, 2)
    t = 0.4 * (q.permute(1, 2, 0, 3) @ k.permute(1, 2, 3, 0))
    if cap:
        t = cap * torch.tanh(t / cap)
    i = torch.arange(s)
    if bias:
        t = t - torch.tensor(slopes)[:, None, None] * (i[:, None] - i).abs()
    seen = (i >= torch.tensor(lo)[:, :, None]) & (i < torch.tensor(hi)[:, :, None])
    t = t.masked_fill(~seen[:, None], -1e30)
    p = torch.softmax(t, -1) * seen.any(-1)[:, None, :, None]
    o = (p @ v.permute(1, 2, 0, 3)).permute(2, 0, 1, 3).reshape(s, b, -1)
    assert np.allclose(ctx, o.detach().numpy())
    want = torch.logsumexp(t, -1).detach().numpy()
    there = np.isfinite(lse)
    assert np.allclose(lse[there], want[there]) and not there[0, :, 9:].any() and there[1].all()
    o.backward(torch.tensor(dctx))
    assert np.allclose(A.backward(dctx, qkv, lo, hi, heads, kv, 0.4, cap, slopes), x.grad.numpy())


def test_hidden_elements_are_not_touched():
    rng = np.random.default_rng(4)
    s, heads, dh = 8, 2, 8
    qkv, dctx = rng.normal(size=(s, 1, 3 * heads * dh)), rng.normal(size=(s, 1, heads * dh))
    ids = np.array([[0]] * 5 + [[1]] * 3)
    lo, hi = A.spans(s, 1, True, 0, ids)
    want = A.forward(qkv, lo, hi, heads, heads, 0.3)[0], A.backward(dctx, qkv, lo, hi, heads, heads, 0.3)
    bad, bad_d = qkv.copy(), dctx.copy()
    bad[5:], bad_d[5:] = np.nan, np.inf
    with np.errstate(invalid="ignore"):
        got = A.forward(bad, lo, hi, heads, heads, 0.3)[0], A.backward(bad_d, bad, lo, hi, heads, heads, 0.3)
    assert np.array_equal(got[0][:5], want[0][:5]) and np.array_equal(got[1][:5], want[1][:5])


@pytest.mark.parametrize("kind", ["silu", "gelu_erf", "gelu_tanh", "sigmoid", "relu"])
def test_gated_block_by_differences_and_against_torch(kind):
    rng = np.random.default_rng(6)
    u, w, w2, b, dy = (rng.normal(size=n) for n in ((7, 5), (5, 12), (6, 5), (12,), (7, 5)))
    z, g = G.forward(kind, u, w, b)
    F = torch.nn.functional
    f = dict(silu=F.silu, gelu_erf=F.gelu, gelu_tanh=lambda a: F.gelu(a, approximate="tanh"), sigmoid=torch.sigmoid, relu=F.relu)[kind]
    t = torch.tensor(u) @ torch.tensor(w) + torch.tensor(b)
    assert np.allclose(g, (f(t[:, :6]) * t[:, 6:]).numpy())
    dz = G.backward(kind, dy, w2, z, b)
    d = rng.normal(size=z.shape)
    loss = lambda x: ((G.act(kind, x[:, :6] + b[:6])[0] * (x[:, 6:] + b[6:])) @ w2 * dy).sum()  # noqa: E731
    assert np.isclose((loss(z + 1e-6 * d) - loss(z - 1e-6 * d)) / 2e-6, (dz * d).sum(), rtol=1e-6)
