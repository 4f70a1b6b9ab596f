"""Attention under spans through the C ABI against fp64.

Tolerances.  bf16: products and sums are fp32; the weights P (and dS) are rounded to bf16 before their product, D = dctx.ctx is made of the
rounded ctx, and the result is rounded: up to three roundings of at most 2^-8 of the value, independent of one another, so at most
sqrt(3) 2^-8 = 0.7e-2 relative in the 2-norm; held to 1e-2 (half of the suite's stated tolerance, with its bounds on rows, columns and
elements).  fp32: hundreds of fp32 operations of 2^-24 each at most, held to 1e-5 (a tenth of the stated one)."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import span_attention as A
from paper_2104_04473_amd import binding as B
from gpu_util import assert_close, dev_bytes, np64, randn, stream, sync, tdt

gpu = pytest.mark.gpu


def packed(s, b, mean, seed, padding=True):
    """Runs of ids, boundaries anywhere; sample 0 may end in padding."""
    rng = np.random.default_rng(seed)
    ids = np.zeros((s, b), dtype=np.int32)
    for j in range(b):
        at, n = 0, int(rng.integers(0, 5))
        while at < s:
            e = min(s, at + int(rng.integers(1, 2 * mean + 1)))
            ids[at:e, j] = n
            at, n = e, int(n == 0)   # neighbouring documents differ, others may share an id
    if padding and s > 2:
        ids[s - max(1, s // 7):, 0] = -1
    return ids


class Rig:
    def __init__(self, dtype, s, b, heads, kv, dh, cap=0.0, bias=False, causal=True, window=0, docs=0, prefix=False, seed=1, scale=None):
        self.cfg = B.make_span_cfg(s, b, heads, kv, dh, dtype, scale=scale, cap=cap)
        self.dtype, self.dims = dtype, (s, b, heads, kv, dh)
        self.qkv, self.dctx = randn((s, b, (heads + 2 * kv) * dh), dtype, seed), randn((s, b, heads * dh), dtype, seed + 1)
        self.slopes = torch.from_numpy(2.0 ** (-8.0 * np.arange(1, heads + 1) / heads)).float().cuda() if bias else None
        self.ids = packed(s, b, docs, seed + 2) if docs else None
        self.prefix = np.random.default_rng(seed).integers(-2, s // 2 + 3, size=(s, b)).astype(np.int32) if prefix else None
        self.lo, self.hi = A.spans(s, b, causal, window, self.ids, self.prefix)
        self.spans = None
        if docs or prefix or window or not causal:
            self.spans = dev_bytes(B.ptdp_attn_spans_bytes(s, b))
            at = [None if a is None else torch.from_numpy(a).cuda() for a in (self.ids, self.prefix)]
            B.check(B.ptdp_attn_spans(int(causal), window, *[None if a is None else a.data_ptr() for a in at], self.spans.data_ptr(), s, b, stream()), "spans")
            sync()
        self.guard = 7.0
        pad = lambda *shape, dt: torch.full((int(np.prod(shape)) + 64,), self.guard, dtype=dt, device="cuda")  # noqa: E731
        self.buffers = dict(ctx=pad(s, b, heads * dh, dt=tdt(dtype)), lse=pad(b, heads, s, dt=torch.float32),
                            dqkv=pad(s, b, (heads + 2 * kv) * dh, dt=tdt(dtype)))
        self.ctx = self.buffers["ctx"][:-64].view(s, b, heads * dh)
        self.lse = self.buffers["lse"][:-64].view(b, heads, s)
        self.dqkv = self.buffers["dqkv"][:-64].view_as(self.qkv)
        self.ws = dev_bytes(B.ptdp_attn_span_workspace_bytes(C.byref(self.cfg)))

    def at(self, t):
        return None if t is None else t.data_ptr()

    def forward(self):
        B.check(B.ptdp_attn_span_fwd(C.byref(self.cfg), self.at(self.qkv), self.at(self.spans), self.at(self.slopes), self.at(self.ctx),
                                     self.at(self.lse), stream()), "span_fwd")

    def backward(self):
        B.check(B.ptdp_attn_span_bwd(C.byref(self.cfg), self.at(self.qkv), self.at(self.spans), self.at(self.slopes), self.at(self.ctx),
                                     self.at(self.lse), self.at(self.dctx), self.at(self.dqkv), self.at(self.ws), stream()), "span_bwd")

    def run(self):
        self.forward()
        self.backward()
        sync()
        for name, t in self.buffers.items():
            assert torch.equal(t[-64:], torch.full_like(t[-64:], self.guard)), name + ": written behind its end"

    def oracle(self):
        s, b, heads, kv, dh = self.dims
        slopes = None if self.slopes is None else np64(self.slopes)
        a = (self.lo, self.hi, heads, kv, float(self.cfg.scale), float(self.cfg.cap), slopes)
        return (*A.forward(np64(self.qkv), *a), A.backward(np64(self.dctx), np64(self.qkv), *a))

    def dense(self):
        """The same as the oracle in torch fp64 on the device, head by head, for long sequences."""
        s, b, heads, kv, dh = self.dims
        x, do = self.qkv.double().view(s, b, heads + 2 * kv, dh), self.dctx.double().view(s, b, heads, dh)
        ctx, lse, grad = torch.zeros_like(do), torch.zeros(b, heads, s, dtype=torch.float64, device="cuda"), torch.zeros_like(x)
        i = torch.arange(s, device="cuda")
        for j in range(b):
            lo, hi = (torch.from_numpy(v[j]).cuda()[:, None] for v in (self.lo, self.hi))
            seen = (i >= lo) & (i < hi)
            some = seen.any(1, keepdim=True)
            for h in range(heads):
                g = heads + h // (heads // kv)
                q, k, v = (x[:, j, n].contiguous() for n in (h, g, g + kv))
                t, d = self.cfg.scale * (q @ k.T), self.cfg.scale
                if self.cfg.cap:
                    th = torch.tanh(t / self.cfg.cap)
                    t, d = self.cfg.cap * th, d * (1 - th * th)
                if self.slopes is not None:
                    t = t - self.slopes[h].double() * (i[:, None] - i).abs()
                t = t.masked_fill(~seen, -float("inf"))
                lse[j, h] = torch.logsumexp(t, 1)
                p = torch.where(some, torch.exp(t - torch.where(some[:, 0], lse[j, h], 0.0)[:, None]), 0.0)
                ctx[:, j, h] = p @ v
                dp = do[:, j, h].contiguous() @ v.T
                dx = p * (dp - (dp * p).sum(1, keepdim=True)) * d
                grad[:, j, h] += dx @ k
                grad[:, j, g] += dx.T @ q
                grad[:, j, g + kv] += p.T @ do[:, j, h].contiguous()
        c = lambda t: t.cpu().numpy()  # noqa: E731
        return c(ctx).reshape(s, b, -1), c(lse), c(grad).reshape(s, b, -1)

    def compare(self, want):
        s, b, heads, kv, dh = self.dims
        ctx, lse, grad = want
        f = 0.5 if self.dtype == B.BF16 else 0.1
        got = np64(self.lse)
        there = np.isfinite(lse)
        assert np.array_equal(there, np.isfinite(got)) and (got[~there] == -np.inf).all()
        # fp32 sums of exact products, the hardware's exponential and logarithm: a few 2^-22, times the scores' size (tens)
        assert np.allclose(got[there], lse[there], rtol=2e-5, atol=2e-5)
        assert_close(np64(self.ctx), ctx, self.dtype, "ctx", factor=f)
        d = np64(self.dqkv)
        assert np.isfinite(d).all()
        cut = (heads * dh, (heads + kv) * dh)
        for name, a, w in zip(("dq", "dk", "dv"), np.split(d, cut, -1), np.split(grad, cut, -1)):
            assert_close(a, w, self.dtype, name, factor=f)
        empty = self.hi <= self.lo
        for j in range(b):   # what sees nothing gets nothing
            assert (np64(self.ctx)[empty[j], j] == 0).all() and (d[empty[j], j, :cut[0]] == 0).all()


SMALL = [  # s, b, heads, kv, dh, options
    (1, 1, 1, 1, 32, {}),
    (1, 3, 2, 1, 64, dict(docs=1)),
    (2, 1, 2, 2, 128, dict(cap=5.0)),
    (31, 2, 3, 3, 96, dict(bias=True)),
    (33, 1, 4, 2, 160, dict(cap=3.0, bias=True)),
    (64, 2, 2, 1, 64, dict(docs=7)),
    (65, 1, 8, 1, 128, dict(docs=20, prefix=True)),
    (97, 2, 2, 2, 32, dict(causal=False)),
    (100, 1, 5, 1, 160, dict(causal=False, docs=30, cap=2.0)),
    (128, 1, 3, 1, 64, dict(window=1)),
    (129, 2, 2, 1, 96, dict(window=40, docs=60)),
    (130, 1, 4, 4, 128, dict(causal=False, window=17, bias=True)),
    (191, 1, 2, 2, 64, dict(prefix=True)),
    (200, 2, 4, 2, 128, dict(docs=50, cap=4.0, bias=True, prefix=True)),
    (257, 1, 2, 1, 160, dict(docs=100)),
]


@gpu
@pytest.mark.parametrize("dtype", [B.BF16, B.F32])
@pytest.mark.parametrize("s,b,heads,kv,dh,options", SMALL)
def test_against_oracle(dtype, s, b, heads, kv, dh, options):
    r = Rig(dtype, s, b, heads, kv, dh, **options)
    r.run()
    r.compare(r.oracle())


@gpu
@pytest.mark.parametrize("s,b,heads,kv,dh,options", [(50, 1, 2, 1, 8, {}), (70, 2, 2, 2, 40, dict(docs=20)), (40, 1, 3, 3, 256, dict(cap=2.0, bias=True)),
                                                     (90, 1, 4, 1, 200, dict(causal=False, window=9))])
def test_fp32_head_sizes(s, b, heads, kv, dh, options):
    r = Rig(B.F32, s, b, heads, kv, dh, **options)
    r.run()
    r.compare(r.oracle())


LONG = [  # enough workgroups for the forms of many, long walks, documents that end inside tiles
    (777, 3, 12, 12, 96, dict(docs=350, prefix=True)),
    (1027, 2, 32, 8, 64, dict(bias=True)),
    (1500, 2, 40, 20, 32, dict(docs=300)),
    (2048, 4, 16, 16, 128, dict(docs=400)),
    (2100, 2, 20, 4, 160, dict(cap=50.0)),
    (1300, 4, 20, 20, 160, dict(docs=500, causal=False)),
    (4096, 1, 16, 1, 128, dict(window=500, cap=30.0)),
    (3001, 1, 8, 8, 64, dict(causal=False, bias=True)),
    (640, 8, 16, 16, 96, dict(docs=90)),
]


@gpu
@pytest.mark.parametrize("s,b,heads,kv,dh,options", LONG)
def test_long(s, b, heads, kv, dh, options):
    r = Rig(B.BF16, s, b, heads, kv, dh, **options)
    r.run()
    r.compare(r.dense())
    first = [t.clone() for t in (r.ctx, r.lse, r.dqkv)]
    r.run()   # and again: the same bits
    assert all(torch.equal(a, t) for a, t in zip(first, (r.ctx, r.lse, r.dqkv)))


FORMS = [  # the other ways that dK and dV are cut up: short rows of many, long rows of many, walks of shared heads in parts
    (300, 8, 16, 16, 128, {}),
    (300, 8, 16, 16, 160, dict(cap=20.0, docs=70)),
    (1100, 2, 16, 16, 128, dict(docs=300)),
    (1100, 2, 16, 16, 160, dict(bias=True)),
    (1100, 4, 16, 16, 32, {}),
    (1100, 4, 16, 16, 96, dict(cap=15.0, prefix=True)),
    (6000, 1, 8, 2, 128, dict(docs=1500)),
    (5000, 1, 16, 4, 64, dict(window=700)),
    (700, 1, 8, 1, 32, dict(docs=9, bias=True)),   # parts without a tile
]


@gpu
@pytest.mark.parametrize("s,b,heads,kv,dh,options", FORMS)
def test_forms_of_key_gradients(s, b, heads, kv, dh, options):
    r = Rig(B.BF16, s, b, heads, kv, dh, **options)
    r.run()
    r.compare(r.dense())
    first = r.dqkv.clone()
    r.run()
    assert torch.equal(first, r.dqkv)


@gpu
@pytest.mark.parametrize("s,b", [(1, 1), (255, 2), (256, 1), (257, 3), (1000, 2), (5000, 1), (9001, 2)])
@pytest.mark.parametrize("causal,window,prefix", [(True, 0, False), (True, 0, True), (False, 0, False), (True, 37, False), (False, 300, False)])
@pytest.mark.parametrize("mean", [1, 40, 3000])
def test_spans(s, b, causal, window, prefix, mean):
    """The integers themselves: a run's first and last token may be thousands of tokens away."""
    ids = packed(s, b, mean, s + mean)
    pre = np.random.default_rng(s).integers(-3, mean + 3, size=(s, b)).astype(np.int32) if prefix else None
    lo, hi = A.spans(s, b, causal, window, ids, pre)
    buf = dev_bytes(B.ptdp_attn_spans_bytes(s, b) + 64).fill_(77)
    at = [None if a is None else torch.from_numpy(a).cuda() for a in (ids, pre)]
    B.check(B.ptdp_attn_spans(int(causal), window, *[None if a is None else a.data_ptr() for a in at], buf.data_ptr(), s, b, stream()), "spans")
    sync()
    assert (buf[B.ptdp_attn_spans_bytes(s, b):] == 77).all()
    got = buf[:s * b * 8].view(torch.int32).view(b, s, 2).cpu().numpy()
    empty = lo >= hi
    assert (got[..., 0][empty] >= got[..., 1][empty]).all()
    assert np.array_equal(got[..., 0][~empty], lo[~empty]) and np.array_equal(got[..., 1][~empty], hi[~empty])


@gpu
@pytest.mark.parametrize("dtype", [B.BF16, B.F32])
@pytest.mark.parametrize("dh,heads,kv", [(64, 2, 1), (128, 4, 4), (160, 2, 2), (96, 2, 1)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_hidden_infinities_reach_nothing(dtype, dh, heads, kv, bad):
    """One document and the padding hold values that are not finite, in q, k, v and dctx: the others' results are the same bits as without (the bf16
    dK and dV, whose keys are made again by another road, within their tolerance)."""
    s, b = 150, 2
    r = Rig(dtype, s, b, heads, kv, dh, cap=5.0, bias=True)
    ids = np.repeat(np.array([0] * 45 + [1] * 20 + [2] * 65 + [-1] * 20, dtype=np.int32)[:, None], b, 1)
    dev = torch.from_numpy(ids).cuda()
    r.spans = dev_bytes(B.ptdp_attn_spans_bytes(s, b))
    B.check(B.ptdp_attn_spans(1, 0, dev.data_ptr(), None, r.spans.data_ptr(), s, b, stream()), "spans")
    r.run()
    want = [t.clone() for t in (r.ctx, r.lse, r.dqkv)]
    gone = torch.from_numpy((ids == 1) | (ids == -1)).cuda()
    r.qkv[gone] = bad
    r.dctx[gone] = bad
    r.run()
    ok = ~gone
    cut = heads * dh if dtype == B.BF16 else r.qkv.shape[2]
    assert torch.equal(r.ctx[ok], want[0][ok]) and torch.equal(r.dqkv[ok][:, :cut], want[2][ok][:, :cut])
    if dtype == B.BF16:
        assert_close(np64(r.dqkv[ok][:, cut:]), np64(want[2][ok][:, cut:]), dtype, "dk, dv", factor=0.5)
    keep = ok[:, 0]
    assert torch.equal(r.lse[:, :, keep], want[1][:, :, keep])
    pad = torch.from_numpy(ids == -1).cuda()
    assert (r.ctx[pad] == 0).all() and (r.dqkv[pad] == 0).all()
    # a document's own values do reach it
    assert not torch.isfinite(r.ctx[torch.from_numpy(ids == 1).cuda()]).any()


@gpu
@pytest.mark.parametrize("dtype", [B.BF16, B.F32])
def test_visible_infinity_reaches_those_that_see_it(dtype):
    """The causal mask: a value that is not finite reaches its own row's successors and nobody before."""
    s, dh = 100, 64
    r = Rig(dtype, s, 1, 2, 2, dh)
    r.run()
    want = r.ctx.clone()
    r.qkv[60, 0, 4 * dh:5 * dh] = float("inf")   # V of head 0
    r.run()
    assert torch.equal(r.ctx[:60], want[:60]) and torch.equal(r.ctx[:, :, dh:], want[:, :, dh:])
    assert not torch.isfinite(r.ctx[60:, :, :dh]).any()


@gpu
@pytest.mark.parametrize("dtype,dh", [(B.BF16, 128), (B.F32, 64)])
def test_gradient_against_differences(dtype, dh):
    """dqkv against differences of sum(ctx * dctx) in fp64 along a random direction (the oracle's forward)."""
    r = Rig(dtype, 40, 1, 4, 2, dh, cap=3.0, bias=True, docs=15)
    r.run()
    s, b, heads, kv, _ = r.dims
    a = (r.lo, r.hi, heads, kv, float(r.cfg.scale), float(r.cfg.cap), np64(r.slopes))
    x, d = np64(r.qkv), np.random.default_rng(0).normal(size=r.qkv.shape)
    f = lambda y: (A.forward(y, *a)[0] * np64(r.dctx)).sum()  # noqa: E731
    want = (f(x + 1e-5 * d) - f(x - 1e-5 * d)) / 2e-5
    got = (np64(r.dqkv) * d).sum()
    # the sum's error: |dqkv's error| |d| / sqrt(n) sqrt(n), at the relative tolerance above
    lim = (1e-2 if dtype == B.BF16 else 1e-5) * np.linalg.norm(np64(r.dqkv)) * 4
    assert abs(got - want) <= lim


@gpu
def test_replayed_and_on_another_stream():
    """Two captured graphs with workspaces of their own, eager work between the replays."""
    rigs = [Rig(B.BF16, 300, 2, 4, 2, 128, docs=80, cap=10.0, seed=k) for k in (1, 50)]
    wants, graphs = [], []
    for r in rigs:
        r.run()
        wants.append([t.clone() for t in (r.ctx, r.lse, r.dqkv)])
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            r.forward()
            r.backward()
        graphs.append(g)
    for _ in range(3):
        for r, g, w in zip(rigs, graphs, wants):
            for t in (r.ctx, r.lse, r.dqkv):
                t.fill_(3.0)
            g.replay()
            sync()
            assert all(torch.equal(a, t) for a, t in zip(w, (r.ctx, r.lse, r.dqkv)))
            r.run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        rigs[0].run()
    side.synchronize()
    assert all(torch.equal(a, t) for a, t in zip(wants[0], (rigs[0].ctx, rigs[0].lse, rigs[0].dqkv)))


def test_refusals():
    """No call that is refused launches anything; pointers are never followed on the host."""
    ok = dict(s=0, b=1, heads=4, kv_heads=2, dh=64, dtype=B.BF16, scale=0.125, cap=0.0)   # s = 0: nothing is touched
    cfg = lambda **k: B.make_span_cfg(**{**ok, **k})  # noqa: E731
    p = 4096

    def fwd(c, *ptrs):
        return B.ptdp_attn_span_fwd(None if c is None else C.byref(c), *(ptrs or (p, None, None, p, p)), None)

    def bwd(c, *ptrs):
        return B.ptdp_attn_span_bwd(None if c is None else C.byref(c), *(ptrs or (p, None, None, p, p, p, 2 * p, p)), None)
    for call in (fwd, bwd):
        assert call(None) == B.E_NULL_PTR and call(cfg()) == B.OK and call(cfg(s=1, b=0)) == B.OK
        for bad in (dict(s=-1), dict(b=-1), dict(heads=0), dict(kv_heads=0), dict(kv_heads=3), dict(dh=0), dict(dh=60), dict(dh=264), dict(dtype=5),
                    dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(cap=-1.0), dict(cap=float("nan")),
                    dict(cap=1e-9), dict(cap=float("inf"))):
            assert call(cfg(**bad)) == B.E_INVALID_ARG, bad
            assert B.ptdp_attn_span_workspace_bytes(C.byref(cfg(**bad))) == 0
        bad = cfg()
        bad.struct_size = 8
        assert call(bad) == B.E_INVALID_ARG
        for bad in (dict(dh=40), dict(dh=256), dict(b=70000), dict(s=2 ** 31 - 1), dict(b=60000, heads=64, kv_heads=64, s=1),
                    dict(heads=1 << 28, kv_heads=1 << 28)):
            assert call(cfg(**bad)) == B.E_UNSUPPORTED, bad
        assert call(cfg(dtype=B.F32, dh=40)) == B.OK and call(cfg(dtype=B.F32, heads=70000, kv_heads=70000, dh=8)) == B.E_UNSUPPORTED
    for k in (0, 3, 4):
        a = [p, None, None, p, p]
        a[k] = None
        assert fwd(cfg(), *a) == B.E_NULL_PTR
    for k in (0, 3, 4, 5, 6, 7):
        a = [p, None, None, p, p, p, 2 * p, p]
        a[k] = None
        assert bwd(cfg(), *a) == B.E_NULL_PTR
    assert fwd(cfg(), p + 8, None, None, p, p) == B.E_INVALID_ARG and fwd(cfg(), p, p + 4, None, p, p) == B.E_INVALID_ARG
    assert bwd(cfg(), p, None, None, p, p, p, p, p) == B.E_INVALID_ARG   # in place
    assert B.ptdp_attn_span_workspace_bytes(C.byref(cfg(s=100, b=3))) >= 4 * 100 * 3 * 4
    spans = lambda *a: B.ptdp_attn_spans(*a, None)  # noqa: E731
    assert spans(1, 0, None, None, p, 0, 1) == B.OK and spans(1, 0, None, None, None, 0, 1) == B.E_NULL_PTR
    for bad in ((2, 0, None, None, p, 0, 1), (1, -1, None, None, p, 0, 1), (0, 0, None, p, p, 0, 1), (1, 5, None, p, p, 0, 1), (1, 0, None, None, p, -1, 1),
                (1, 0, None, None, p, 0, -1), (1, 0, None, None, p + 4, 0, 1)):
        assert spans(*bad) == B.E_INVALID_ARG, bad
    assert spans(1, 0, None, None, p, 1, 70000) == B.E_UNSUPPORTED and B.ptdp_attn_spans_bytes(-1, 1) == 0 and B.ptdp_attn_spans_bytes(1, 70000) == 0
    assert B.ptdp_attn_spans_bytes(33, 2) == 33 * 2 * 8 + 2 * 2 * 16


@pytest.mark.parametrize("dtype", [B.BF16, B.F32])
def test_workspace_bytes(dtype):
    """Statistics of every query, and sums of dK and dV where few key blocks of shared heads are walked in parts: at most one set for each query head."""
    for s, b, heads, kv, dh in ((0, 1, 4, 2, 64), (1, 0, 4, 2, 64), (1, 1, 4, 1, 64), (33, 2, 8, 8, 128), (2048, 1, 16, 2, 128), (16384, 1, 8, 2, 128)):
        n = B.ptdp_attn_span_workspace_bytes(C.byref(B.make_span_cfg(s, b, heads, kv, dh, dtype)))
        rows = (s + 31) // 32 * 32 * b * heads
        least = s * b * heads * (8 if dtype == B.BF16 else 4)
        assert least <= n <= rows * 8 + (heads > kv) * rows * 2 * dh * 4 + 256, (s, b, heads, kv, dh, n)
