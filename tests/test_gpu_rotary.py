"""Rotary positions through the C ABI against the fp64 oracle.

Tolerances: a result is (c x - n y) rounded once.  fp32: c and n are off by a few 2^-24 of the amplitude (the angle's fraction of a
turn is rounded to fp32: at most 2^-25 turns, 2^-25 * 2 pi < 2^-22 radians), and three fp32 operations follow: below 2^-20 of
amplitude * |pair|.  bf16: that and one rounding of at most 2^-8 of the result."""
import numpy as np
import pytest
import torch

from oracle import rotary as R
from paper_2104_04473_amd import binding as B
from gpu_util import np64, randn, stream, sync

gpu = pytest.mark.gpu

CASES = [  # dtype, layout, s, b, heads, kv heads, dh, rot, positions
    (B.BF16, B.ROTARY_HALVES, 1, 1, 1, 1, 8, 8, None),
    (B.BF16, B.ROTARY_HALVES, 33, 3, 4, 2, 64, 64, None),
    (B.BF16, B.ROTARY_HALVES, 7, 2, 5, 5, 128, 64, "far"),
    (B.BF16, B.ROTARY_HALVES, 9, 1, 3, 1, 96, 96, "any"),
    (B.BF16, B.ROTARY_HALVES, 5, 2, 2, 1, 40, 24, "any"),      # halves of 12: no whole number of 16 bytes
    (B.BF16, B.ROTARY_HALVES, 3, 1, 40, 8, 256, 256, "far"),
    (B.BF16, B.ROTARY_PAIRS, 65, 1, 20, 4, 160, 160, None),
    (B.BF16, B.ROTARY_PAIRS, 11, 2, 1, 1, 8, 8, "any"),
    (B.BF16, B.ROTARY_PAIRS, 6, 1, 9, 3, 256, 200, "far"),
    (B.F32, B.ROTARY_HALVES, 17, 2, 4, 4, 64, 32, None),
    (B.F32, B.ROTARY_HALVES, 4, 1, 3, 1, 24, 24, "any"),
    (B.F32, B.ROTARY_HALVES, 2, 1, 2, 2, 256, 256, "far"),
    (B.F32, B.ROTARY_PAIRS, 19, 3, 6, 2, 80, 80, "far"),
    (B.F32, B.ROTARY_PAIRS, 2, 2, 8, 1, 256, 256, "any"),
    (B.F32, B.ROTARY_PAIRS, 1, 1, 1, 1, 16, 8, None),
]


def place(kind, s, b, seed=5):
    """Positions: far into a context, or any 32-bit value."""
    if kind is None:
        return None
    rng = np.random.default_rng(seed)
    p = rng.integers(1 << 20, 1 << 24, size=(s, b)) if kind == "far" else rng.integers(-(1 << 31), 1 << 31, size=(s, b))
    if kind == "any":
        p[0, 0] = -(1 << 31)
    return p.astype(np.int32)


def call(fn, dtype, layout, x, pos, turns, out, heads, kv, dh, rot, amp):
    s, b = x.shape[:2]
    return fn(dtype, layout, x.data_ptr(), None if pos is None else pos.data_ptr(), turns.data_ptr(), out.data_ptr(), s, b, heads, kv, dh, rot,
              amp, stream())


@gpu
@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("dtype,layout,s,b,heads,kv,dh,rot,kind", CASES)
def test_rotary(dtype, layout, s, b, heads, kv, dh, rot, kind, back):
    f = B.rotary_turns(rot, scaling=B.ROTARY_RAMP, factor=8.0, trained=4096, slow=1.0, fast=32.0)
    turns = torch.tensor(f, dtype=torch.float64, device="cuda")
    x = randn((s, b, (heads + 2 * kv) * dh), dtype, 3)
    p = place(kind, s, b)
    pos = None if p is None else torch.from_numpy(p).cuda()
    amp = 1.25
    fn = B.ptdp_rotary_bwd if back else B.ptdp_rotary_fwd
    guard = torch.full((s * b * x.shape[2] + 64,), 7.0, dtype=x.dtype, device="cuda")   # rows behind the last one stay as they were
    out = guard[:x.numel()].view_as(x)
    B.check(call(fn, dtype, layout, x, pos, turns, out, heads, kv, dh, rot, amp), "rotary")
    same = x.clone()
    B.check(call(fn, dtype, layout, same, pos, turns, same, heads, kv, dh, rot, amp), "rotary in place")
    sync()
    assert torch.equal(out, same)
    assert torch.equal(guard[x.numel():], torch.full((64,), 7.0, dtype=x.dtype, device="cuda"))
    xs = np64(x)
    want = R.rotate(xs, p, np.array(f), heads, kv, rot, layout == B.ROTARY_PAIRS, amp, back)
    got = np64(out)
    size = amp * (np.abs(xs) + np.abs(R.rotate(xs, np.full((s, b), 1), np.full(rot // 2, 0.25), heads, kv, rot, layout == B.ROTARY_PAIRS)))  # |x| + |y|
    assert (np.abs(got - want) <= 2.0 ** -20 * size + (2.0 ** -8 * np.abs(want) if dtype == B.BF16 else 0)).all()
    rest = np.ones((heads + 2 * kv, dh), dtype=bool)
    rest[:heads + kv, :rot] = False
    assert np.array_equal(got[..., rest.ravel()], xs[..., rest.ravel()])


@gpu
@pytest.mark.parametrize("dtype", [B.BF16, B.F32])
def test_rotary_replayed(dtype):
    """Captured with eager calls between the replays; a stream other than the current one."""
    heads, kv, dh = 8, 2, 64
    x = randn((130, 2, (heads + 2 * kv) * dh), dtype, 9)
    turns = torch.tensor(B.rotary_turns(dh), dtype=torch.float64, device="cuda")
    want, out = torch.empty_like(x), torch.empty_like(x)
    B.check(call(B.ptdp_rotary_fwd, dtype, 0, x, None, turns, want, heads, kv, dh, dh, 1.0), "rotary")
    sync()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.check(call(B.ptdp_rotary_fwd, dtype, 0, x, None, turns, out, heads, kv, dh, dh, 1.0), "rotary")
    for _ in range(3):
        out.fill_(3.0)
        graph.replay()
        sync()
        assert torch.equal(out, want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        out.zero_()
        B.check(call(B.ptdp_rotary_fwd, dtype, 0, x, None, turns, out, heads, kv, dh, dh, 1.0), "rotary")
    side.synchronize()
    assert torch.equal(out, want)


def test_turns_are_the_oracles():
    for rot in (8, 64, 160, 256):
        for name, scaling in (("plain", B.ROTARY_PLAIN), ("linear", B.ROTARY_LINEAR), ("base", B.ROTARY_BASE), ("ramp", B.ROTARY_RAMP)):
            got = B.rotary_turns(rot, 50000.0, scaling, 4.0, 2048, 1.0, 32.0)
            assert np.allclose(got, R.turns(rot, 50000.0, name, 4.0, 2048, 1.0, 32.0), rtol=1e-14, atol=0)


def test_refusals():
    import ctypes as C
    out = (C.c_double * 128)()
    ok = dict(rot=64, base=1e4, scaling=B.ROTARY_RAMP, factor=2.0, trained=2048.0, slow=1.0, fast=32.0)
    turns = lambda **k: B.ptdp_rotary_turns(*[{**ok, **k}[n] for n in ok], out)  # noqa: E731
    assert turns() == B.OK and B.ptdp_rotary_turns(*ok.values(), None) == B.E_NULL_PTR
    for bad in (dict(rot=0), dict(rot=12), dict(rot=264), dict(base=0.0), dict(base=-1.0), dict(base=float("nan")), dict(scaling=4), dict(scaling=-1),
                dict(factor=0.0), dict(factor=float("inf")), dict(trained=0.0), dict(slow=-1.0), dict(slow=32.0), dict(fast=float("nan"))):
        assert turns(**bad) == B.E_INVALID_ARG, bad
    assert turns(scaling=B.ROTARY_PLAIN, factor=0.0, trained=-1.0, slow=5.0, fast=5.0) == B.OK   # not used
    ok = dict(dtype=B.BF16, layout=0, x=16, pos=None, turns=16, out=16, s=0, b=1, heads=4, kv=2, dh=64, rot=32, amp=1.0)   # s = 0: nothing is touched
    call = lambda fn, **k: fn(*[{**ok, **k}[n] for n in ok], None)  # noqa: E731
    for fn in (B.ptdp_rotary_fwd, B.ptdp_rotary_bwd):
        assert call(fn) == B.OK and call(fn, s=1, b=0) == B.OK
        for bad in (dict(dtype=2), dict(layout=2), dict(s=-1), dict(b=-1), dict(heads=0), dict(kv=0), dict(kv=3), dict(dh=0), dict(dh=60), dict(dh=264),
                    dict(rot=0), dict(rot=72), dict(rot=12), dict(amp=float("inf")), dict(amp=float("nan")), dict(x=8), dict(out=18), dict(turns=8)):
            assert call(fn, **bad) == B.E_INVALID_ARG, bad
        for null in ("x", "turns", "out"):
            assert call(fn, **{null: None}) == B.E_NULL_PTR
        assert call(fn, s=1 << 30, b=4) == B.E_UNSUPPORTED
        assert call(fn, heads=1 << 29, kv=1 << 29) == B.E_UNSUPPORTED
