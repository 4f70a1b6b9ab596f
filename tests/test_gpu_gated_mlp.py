"""The gated feed-forward block's products through the C ABI against fp64.

Tolerances.  bf16: products of bf16 values are exact in fp32, the sums are fp32; z, g and dz are rounded once, by at most 2^-8 of the value, or
(where a call takes 256 x 256 tiles) dz twice: held to 2^-8 and sqrt(2) 2^-8, rounded up: 0.4e-2 and 0.6e-2 in the relative 2-norm.  dbias sums
fp32 values; where dg has been rounded once, its relative error is at most 2^-8 as well (and averages out).  fp32: k 2^-24 at most for sums of k = 2048 in any
order, 1.2e-4 in theory and sqrt(k) 2^-24 = 3e-6 for independent roundings; held to 1e-5 (a tenth of the suite's stated tolerance)."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import gated_mlp as G
from paper_2104_04473_amd import binding as B
from gpu_util import assert_close, dev_bytes, np64, randn, stream, sync, tdt

gpu = pytest.mark.gpu
GATES = dict(silu=B.GATE_SILU, gelu_erf=B.GATE_GELU_ERF, gelu_tanh=B.GATE_GELU_TANH, sigmoid=B.GATE_SIGMOID, relu=B.GATE_RELU)


def act64(kind, a):
    """f(a) and f'(a) on the device in fp64 (by differentiation)."""
    F = torch.nn.functional
    a = a.clone().requires_grad_(True)
    f = dict(silu=F.silu, gelu_erf=F.gelu, gelu_tanh=lambda x: F.gelu(x, approximate="tanh"), sigmoid=torch.sigmoid, relu=F.relu)[kind](a)
    return f.detach(), torch.autograd.grad(f.sum(), a)[0]


class Rig:
    def __init__(self, dtype, rows, width, inner, bias, seed=1):
        self.dtype, self.size = dtype, (rows, width, inner)
        self.u, self.w = randn((rows, width), dtype, seed), randn((width, 2 * inner), dtype, seed + 1, scale=width ** -0.5)
        self.dy, self.w2 = randn((rows, width), dtype, seed + 2), randn((inner, width), dtype, seed + 3, scale=width ** -0.5)
        self.bias = randn((2 * inner,), dtype, seed + 4, scale=0.5) if bias else None
        pad = lambda n, dt: torch.full((n + 64,), 7.0, dtype=dt, device="cuda")  # noqa: E731
        self.guards = [pad(rows * 2 * inner, tdt(dtype)), pad(rows * inner, tdt(dtype)), pad(rows * 2 * inner, tdt(dtype))]
        self.z, self.g, self.dz = (t[:-64].view(rows, -1) for t in self.guards)
        self.dbias = torch.full((2 * inner,), 0.25, device="cuda") if bias else None
        self.ws = dev_bytes(B.ptdp_gated_mlp_workspace_bytes(dtype, rows, width, inner))

    def at(self, t):
        return None if t is None else t.data_ptr()

    def forward(self, kind):
        B.check(B.ptdp_gated_mlp_fwd(self.dtype, GATES[kind], self.at(self.u), self.at(self.w), self.at(self.bias), self.at(self.z), self.at(self.g),
                                     *self.size, stream()), "gated_mlp_fwd")

    def backward(self, kind, dz=None):
        B.check(B.ptdp_gated_mlp_bwd(self.dtype, GATES[kind], self.at(self.dy), self.at(self.w2), self.at(self.z), self.at(self.bias),
                                     self.at(self.dz if dz is None else dz), self.at(self.dbias), self.at(self.ws), *self.size, stream()), "gated_mlp_bwd")

    def check(self, kind):
        rows, width, inner = self.size
        self.forward(kind)
        self.backward(kind)
        sync()
        for t in self.guards:
            assert (t[-64:] == 7.0).all(), "written behind its end"
        f = 0.2 if self.dtype == B.BF16 else 0.1
        z = self.u.double() @ self.w.double()
        b = 0.0 if self.bias is None else self.bias.double()
        x = z + b
        c = lambda t: t.cpu().numpy()  # noqa: E731
        assert_close(np64(self.z), c(z), self.dtype, "z", factor=f)
        assert_close(np64(self.g), c(act64(kind, x[:, :inner])[0] * x[:, inner:]), self.dtype, "g", factor=f)
        x = self.z.double() + b   # the backward starts from z as it is stored
        v, d = act64(kind, x[:, :inner])
        dg = self.dy.double() @ self.w2.double().T
        dz = torch.cat((dg * d * x[:, inner:], dg * v), 1)
        assert_close(np64(self.dz), c(dz), self.dtype, "dz", factor=1.5 * f)
        if self.bias is not None:
            got, want = np64(self.dbias) - 0.25, c(dz.sum(0))
            # rounded dg: 2^-8 of each summand, of random sign; the sums are sqrt(rows) times a summand
            lim = (2.0 ** -8 if self.dtype == B.BF16 else 1e-5) * c(dz.abs().square().sum(0).sqrt()) * 4 + 1e-5
            assert (np.abs(got - want) <= lim).all()
        before = self.dz.clone()
        self.backward(kind, self.z)   # in place, with the same bits
        sync()
        assert torch.equal(self.z, before)


@gpu
@pytest.mark.parametrize("dtype", [B.BF16, B.F32])
@pytest.mark.parametrize("kind", sorted(GATES))
@pytest.mark.parametrize("rows,width,inner,bias", [(1, 8, 8, True), (3, 72, 40, False), (65, 128, 72, True), (130, 264, 136, True)])
def test_small(dtype, kind, rows, width, inner, bias):
    Rig(dtype, rows, width, inner, bias).check(kind)


# the forms of the bf16 kernels: (forward, backward) tiles and groups of waves, asserted below
FORMS = [(1998, 2048, 5504), (2048, 4096, 2816), (66, 512, 1368), (513, 1024, 1024), (700, 640, 4096), (300, 2000, 600), (1, 4096, 11008), (4000, 512, 512),
         (1030, 4096, 4104), (129, 8192, 904), (64, 64, 16384), (2048, 1024, 1408), (520, 512, 2056), (1024, 3000, 2816), (16, 12288, 6144), (900, 200, 2400), (1500, 2328, 3168), (2048, 656, 6240),
         (80, 472, 9000), (270, 392, 18000)]


def form(back, rows, width, inner):
    v = [C.c_int() for _ in range(3)]
    B.check(B.ptdp_gated_mlp_form(back, rows, width, inner, *[C.byref(x) for x in v]), "form")
    return tuple(x.value for x in v)


def test_every_form_is_run():
    every = {(256, 256, 1), (128, 128, 1), (128, 128, 2), (128, 64, 2), (64, 64, 2), (128, 64, 1), (256, 128, 2), (256, 192, 1)}
    for back in (0, 1):
        assert {form(back, *size) for size in FORMS} == every


@gpu
@pytest.mark.parametrize("rows,width,inner", FORMS)
def test_forms(rows, width, inner):
    for k, (kind, bias) in enumerate((("silu", True), ("gelu_tanh", False))):
        Rig(B.BF16, rows, width, inner, bias, seed=10 * k).check(kind)


@gpu
@pytest.mark.parametrize("rows,width,inner", [(640, 512, 1368), (1500, 1024, 2816)])
def test_fp32(rows, width, inner):
    Rig(B.F32, rows, width, inner, True).check("gelu_erf")


@gpu
@pytest.mark.parametrize("kind", sorted(GATES))
def test_against_the_oracle_and_its_gradient(kind):
    r = Rig(B.F32, 20, 16, 24, True)
    r.forward(kind)
    r.backward(kind)
    sync()
    z, g = G.forward(kind, np64(r.u), np64(r.w), np64(r.bias))
    assert_close(np64(r.z), z, B.F32, "z", factor=0.1)
    assert_close(np64(r.g), g, B.F32, "g", factor=0.1)
    assert_close(np64(r.dz), G.backward(kind, np64(r.dy), np64(r.w2), np64(r.z), np64(r.bias)), B.F32, "dz", factor=0.1)


@gpu
def test_large_and_infinite_arguments():
    """Activations far out, and sums that are not finite: as the formulas have them."""
    r = Rig(B.BF16, 8, 8, 8, False)
    r.u.zero_()
    r.u[:, 0] = torch.tensor([0.0, 1e4, -1e4, 3e38, -3e38, 200.0, -200.0, float("inf")], device="cuda").bfloat16()
    r.w.zero_()
    r.w[0] = 1.0
    for kind in GATES:
        r.forward(kind)
        sync()
        a = np64(r.u)[:7, 0]
        with np.errstate(over="ignore", invalid="ignore"):
            want = np.array([0.0 if kind != "sigmoid" else a[0] * 0.5] + [float(torch.tensor(x).sigmoid() * x) if kind == "sigmoid" else max(x, 0.0) * x
                                                                           for x in a[1:]])
        got = np64(r.g)[:7, 0]
        fin = np.abs(want) <= float(torch.finfo(torch.bfloat16).max)   # beyond: rounded to infinity
        assert np.allclose(got[fin], want[fin], rtol=2.0 ** -8, atol=1e-30) and np.isinf(got[~fin]).all(), (kind, got, want)


@gpu
def test_replayed_and_on_another_stream():
    rigs = [Rig(B.BF16, 300, 512, 1000, True), Rig(B.BF16, 2048, 512, 4096, True)]
    for r in rigs:
        r.forward("silu")
        r.backward("silu")
        sync()
        want = [t.clone() for t in (r.z, r.g, r.dz, r.dbias)]
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            r.forward("silu")
            r.backward("silu")
        for _ in range(3):
            for t in (r.z, r.g, r.dz):
                t.fill_(3.0)
            r.dbias.fill_(0.25)
            graph.replay()
            sync()
            assert all(torch.equal(a, t) for a, t in zip(want, (r.z, r.g, r.dz, r.dbias)))
            r.forward("relu")   # the program's own work between the replays
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            r.dbias.fill_(0.25)
            r.forward("silu")
            r.backward("silu")
        side.synchronize()
        assert all(torch.equal(a, t) for a, t in zip(want, (r.z, r.g, r.dz, r.dbias)))


def test_refusals():
    p = 4096
    ok = dict(dtype=B.BF16, gate=0, u=p, w=p, bias=None, z=p, g=p, rows=0, width=64, inner=64)   # rows = 0: nothing is touched
    fwd = lambda **k: B.ptdp_gated_mlp_fwd(*[{**ok, **k}[n] for n in ok], None)  # noqa: E731
    okb = dict(dtype=B.BF16, gate=0, dy=p, w2=p, z=p, bias=None, dz=p, dbias=None, ws=p, rows=0, width=64, inner=64)
    bwd = lambda **k: B.ptdp_gated_mlp_bwd(*[{**okb, **k}[n] for n in okb], None)  # noqa: E731
    for call in (fwd, bwd):
        assert call() == B.OK
        for bad in (dict(dtype=2), dict(gate=-1), dict(gate=5), dict(rows=-1), dict(width=0), dict(width=60), dict(inner=0), dict(inner=-8), dict(inner=60),
                    dict(z=p + 8), dict(bias=p + 2)):
            assert call(**bad) == B.E_INVALID_ARG, bad
        for big in (dict(rows=1 << 24, width=64), dict(width=1 << 16, inner=1 << 14), dict(width=8, inner=1 << 21), dict(rows=1 << 22, width=8, inner=1 << 13)):
            assert call(**big) == B.E_UNSUPPORTED, big
    for null in ("u", "w", "z", "g"):
        assert fwd(**{null: None}) == B.E_NULL_PTR
    for null in ("dy", "w2", "z", "dz", "ws"):
        assert bwd(**{null: None}) == B.E_NULL_PTR
    assert B.ptdp_gated_mlp_workspace_bytes(B.BF16, 64, 60, 64) == 0 and B.ptdp_gated_mlp_workspace_bytes(B.BF16, 64, 64, 64) > 0
    v = [C.byref(C.c_int()) for _ in range(3)]
    assert B.ptdp_gated_mlp_form(0, 64, 64, 64, *v) == B.OK and B.ptdp_gated_mlp_form(2, 64, 64, 64, *v) == B.E_INVALID_ARG
    assert B.ptdp_gated_mlp_form(1, 0, 64, 64, *v) == B.E_INVALID_ARG and B.ptdp_gated_mlp_form(1, 64, 64, 64, None, v[1], v[2]) == B.E_NULL_PTR
    assert fwd(dtype=B.F32, width=1 << 15, inner=1 << 13) == B.E_UNSUPPORTED and fwd(dtype=B.F32) == B.OK
