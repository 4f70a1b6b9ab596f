"""The operators of later GPT-style layers run together, as a layer runs them: the QKV product, rotary positions, attention under spans, the output
product, the gated feed-forward block, and back to the gradients of the input and of all weights.

Tolerance: the suite's stated one.  bf16: from x to its gradient a value is rounded at most fourteen times (qkv, its rotation, P, ctx, u, z, g; dz, du,
dctx, dS, dqkv, its rotation, dx), each time by 2^-8 / sqrt(3) relative in the 2-norm at most, independently: sqrt(14 / 3) 2^-8 = 0.85e-2, with scores
of order one (nothing enlarges an error), less than half of 2e-2.  fp32: sums of hundreds of products, 2^-24 each, held to 1e-4."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import gated_mlp as G
from oracle import rotary as R
from oracle import span_attention as A
from paper_2104_04473_amd import binding as B
from gpu_util import assert_close, dev_bytes, np64, randn, stream, sync, tdt

gpu = pytest.mark.gpu


class Layer:
    """x -> qkv = x a -> turned -> ctx -> u = ctx o -> y = gated(u); every buffer allocated once."""

    def __init__(self, dtype, s, b, heads, kv, dh, inner, rot, cap, bias, seed):
        self.dtype, self.dims, self.rot = dtype, (s, b, heads, kv, dh), rot
        h, row = heads * dh, (heads + 2 * kv) * dh
        self.T, self.h, self.row, self.inner = s * b, h, row, inner
        new = lambda *shape, dt=None: torch.empty(shape, dtype=dt or tdt(dtype), device="cuda")  # noqa: E731
        self.x, self.dy = randn((s, b, h), dtype, seed), randn((s, b, h), dtype, seed + 1)
        self.weights = {n: randn(sh, dtype, seed + 2 + k, scale=sh[0] ** -0.5)
                        for k, (n, sh) in enumerate(dict(a=(h, row), o=(h, h), w=(h, 2 * inner), w2=(inner, h)).items())}
        self.bias = randn((2 * inner,), dtype, seed + 9)
        self.ids = np.repeat((np.arange(s) // 37).astype(np.int32)[:, None], b, 1)
        self.ids[s - 5:, 0] = -1
        self.where = np.random.default_rng(seed).integers(0, 5000, size=(s, b)).astype(np.int32)
        self.freq = B.rotary_turns(rot)
        self.dev = [torch.from_numpy(self.ids).cuda(), torch.from_numpy(self.where).cuda(), torch.tensor(self.freq, dtype=torch.float64, device="cuda")]
        self.slopes = torch.from_numpy(2.0 ** -np.arange(1, heads + 1)).float().cuda() if bias else None
        self.cfg = B.make_span_cfg(s, b, heads, kv, dh, dtype, cap=cap)
        self.spans = dev_bytes(B.ptdp_attn_spans_bytes(s, b))
        self.qkv, self.dqkv, self.ctx, self.lse = new(s, b, row), new(s, b, row), new(s, b, h), new(b, heads, s, dt=torch.float32)
        self.u, self.z, self.g, self.y = new(s, b, h), new(s, b, 2 * inner), new(s, b, inner), new(s, b, h)
        self.du, self.dctx, self.dx = new(s, b, h), new(s, b, h), new(s, b, h)
        self.grads = {n: torch.zeros(t.shape, device="cuda") for n, t in self.weights.items()}
        self.dbias = torch.zeros(2 * inner, device="cuda")
        self.ws = dev_bytes(max(B.ptdp_attn_span_workspace_bytes(C.byref(self.cfg)), B.ptdp_gated_mlp_workspace_bytes(dtype, self.T, h, inner)))

    def product(self, mode, a, b, c, M, N, K, gradient=False):
        B.check(B.ptdp_gemm(self.dtype, mode, a.data_ptr(), b.data_ptr(), c.data_ptr(), None, M, N, K, int(gradient), int(gradient), None, 0, stream()), "gemm")

    def run(self):
        s, b, heads, kv, dh = self.dims
        T, h, row, inner, p = self.T, self.h, self.row, self.inner, lambda t: None if t is None else t.data_ptr()
        ids, where, freq = self.dev
        for t in (*self.grads.values(), self.dbias):
            t.zero_()
        rows, cfg = (s, b, heads, kv, dh, self.rot), C.byref(self.cfg)
        B.check(B.ptdp_attn_spans(1, 0, p(ids), None, p(self.spans), s, b, stream()), "spans")
        self.product(B.GEMM_NN, self.x, self.weights["a"], self.qkv, T, row, h)
        B.check(B.ptdp_rotary_fwd(self.dtype, B.ROTARY_HALVES, p(self.qkv), p(where), p(freq), p(self.qkv), *rows, 1.0, stream()), "rotary_fwd")
        B.check(B.ptdp_attn_span_fwd(cfg, p(self.qkv), p(self.spans), p(self.slopes), p(self.ctx), p(self.lse), stream()), "span_fwd")
        self.product(B.GEMM_NN, self.ctx, self.weights["o"], self.u, T, h, h)
        B.check(B.ptdp_gated_mlp_fwd(self.dtype, B.GATE_SILU, p(self.u), p(self.weights["w"]), p(self.bias), p(self.z), p(self.g), T, h, inner, stream()), "fwd")
        self.product(B.GEMM_NN, self.g, self.weights["w2"], self.y, T, h, inner)

        self.product(B.GEMM_TN, self.g, self.dy, self.grads["w2"], inner, h, T, True)
        B.check(B.ptdp_gated_mlp_bwd(self.dtype, B.GATE_SILU, p(self.dy), p(self.weights["w2"]), p(self.z), p(self.bias), p(self.z), p(self.dbias), p(self.ws),
                                     T, h, inner, stream()), "bwd")   # dz in place of z
        self.product(B.GEMM_TN, self.u, self.z, self.grads["w"], h, 2 * inner, T, True)
        self.product(B.GEMM_NT, self.z, self.weights["w"], self.du, T, h, 2 * inner)
        self.product(B.GEMM_TN, self.ctx, self.du, self.grads["o"], h, h, T, True)
        self.product(B.GEMM_NT, self.du, self.weights["o"], self.dctx, T, h, h)
        B.check(B.ptdp_attn_span_bwd(cfg, p(self.qkv), p(self.spans), p(self.slopes), p(self.ctx), p(self.lse), p(self.dctx), p(self.dqkv), p(self.ws),
                                     stream()), "span_bwd")
        B.check(B.ptdp_rotary_bwd(self.dtype, B.ROTARY_HALVES, p(self.dqkv), p(where), p(freq), p(self.dqkv), *rows, 1.0, stream()), "rotary_bwd")
        self.product(B.GEMM_TN, self.x, self.dqkv, self.grads["a"], h, row, T, True)
        self.product(B.GEMM_NT, self.dqkv, self.weights["a"], self.dx, T, h, row)

    def results(self):
        return dict(y=self.y, dx=self.dx, dbias=self.dbias, **{"d" + n: t for n, t in self.grads.items()})

    def oracle(self):
        s, b, heads, kv, dh = self.dims
        x, dy, w = np64(self.x), np64(self.dy), {n: np64(t) for n, t in self.weights.items()}
        flat = lambda t: t.reshape(-1, t.shape[-1])  # noqa: E731
        turn = lambda t, back: R.rotate(t, self.where, np.array(self.freq), heads, kv, self.rot, False, back=back)  # noqa: E731
        lo, hi = A.spans(s, b, True, 0, self.ids, None)
        a = (lo, hi, heads, kv, float(self.cfg.scale), float(self.cfg.cap), None if self.slopes is None else np64(self.slopes))
        qkv = turn(x @ w["a"], False)
        ctx, _ = A.forward(qkv, *a)
        u = ctx @ w["o"]
        z, g = G.forward("silu", u, w["w"], np64(self.bias))
        dz = G.backward("silu", dy, w["w2"], z, np64(self.bias))
        du = dz @ w["w"].T
        dqkv = turn(A.backward(du @ w["o"].T, qkv, *a), True)
        return dict(y=g @ w["w2"], dx=dqkv @ w["a"].T, dbias=flat(dz).sum(0), da=flat(x).T @ flat(dqkv), do=flat(ctx).T @ flat(du),
                    dw=flat(u).T @ flat(dz), dw2=flat(g).T @ flat(dy))


@gpu
@pytest.mark.parametrize("dtype", [B.BF16, B.F32])
@pytest.mark.parametrize("s,b,heads,kv,dh,inner,rot,cap,bias", [(132, 2, 4, 2, 64, 320, 64, 0.0, False), (72, 1, 2, 1, 128, 200, 48, 6.0, True),
                                                                (72, 3, 5, 1, 32, 64, 32, 4.0, False)])
def test_layer_against_oracle_and_replayed(dtype, s, b, heads, kv, dh, inner, rot, cap, bias):
    r = Layer(dtype, s, b, heads, kv, dh, inner, rot, cap, bias, 7)
    r.run()
    sync()
    eager = {n: t.clone() for n, t in r.results().items()}
    for n, want in r.oracle().items():
        assert_close(np64(eager[n]), want, dtype, n, local=n != "dbias")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r.run()
    for _ in range(3):
        for t in r.results().values():
            t.fill_(5.0)
        graph.replay()
        sync()
        assert all(torch.equal(t, eager[n]) for n, t in r.results().items())
        r.run()   # eager work between the replays
        sync()
