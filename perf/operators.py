"""The operators of later GPT-style layers, as cases for timing: rotary positions, attention under spans with capped scores,
a distance bias and shared key/value heads, and the gated feed-forward block's fused products.

A case is a dict of plain values.  Its `op` says which operator one pass goes through:

  rotary     `back` False: rotation of Q and K in rows of Q | K | V; True: of their gradients
  attention  `back` False: forward; True: a training step, forward and backward
  gate       `back` False: z = u w and g = act(z_gate + b) (z_up + b); True: dz and the bias gradient from dy

With `own` false `run` is the plain form: elementary torch operations in 32 bits (angles in 64), rounded once at the end.
"""
import ctypes as C
import math

import numpy as np
import torch

own = False
DEV = "cuda:0"


def listed():
    return [
        # one short sequence of a small model: a launch and little else
        dict(name="rotary 64 tokens", op="rotary", back=False, dtype="bf16", s=64, b=1, heads=8, kv=8, dh=64, rot=64, pairs=False,
             scaling="plain", places=False),
        # a microbatch of an unsharded mid-size model
        dict(name="rotary 2048 b4", op="rotary", back=False, dtype="bf16", s=2048, b=4, heads=16, kv=16, dh=128, rot=128, pairs=False,
             scaling="plain", places=False),
        # gradients of a long row of packed documents whose positions start again, part of each head rotated, scaled beyond the trained length
        dict(name="rotary long fp32 back", op="rotary", back=True, dtype="fp32", s=30011, b=1, heads=20, kv=4, dh=160, rot=64, pairs=True,
             scaling="ramp", places=True),
        # the smallest training configuration, with a cap
        dict(name="attn fp32 capped", op="attention", back=True, dtype="fp32", s=128, b=2, heads=4, kv=4, dh=64, cap=30.0, bias=False,
             causal=True, docs=0, prefix=False, window=0),
        # pretraining on packed documents, their boundaries anywhere
        dict(name="attn documents", op="attention", back=True, dtype="bf16", s=2048, b=4, heads=16, kv=16, dh=128, cap=0.0, bias=False,
             causal=True, docs=400, prefix=False, window=0),
        # a shard of a wide model, capped scores, key/value heads shared by five
        dict(name="attn capped 4096", op="attention", back=True, dtype="bf16", s=4096, b=1, heads=20, kv=4, dh=160, cap=50.0, bias=False,
             causal=True, docs=0, prefix=False, window=0),
        # evaluation with a distance bias on a length that fills no tile
        dict(name="attn distance forward", op="attention", back=False, dtype="bf16", s=1027, b=2, heads=32, kv=8, dh=64, cap=0.0, bias=True,
             causal=True, docs=0, prefix=False, window=0),
        # prompts read both ways, answers from left to right
        dict(name="attn prefix", op="attention", back=True, dtype="bf16", s=777, b=3, heads=12, kv=12, dh=96, cap=0.0, bias=False,
             causal=True, docs=350, prefix=True, window=0),
        # training at a long context: long documents, shared heads, bias
        dict(name="attn long documents", op="attention", back=True, dtype="bf16", s=16384, b=1, heads=8, kv=2, dh=128, cap=0.0, bias=True,
             causal=True, docs=6000, prefix=False, window=0),
        # development runs in fp32
        dict(name="gate fp32 ragged", op="gate", back=False, dtype="fp32", rows=66, width=512, inner=1368, act="gelu_tanh", bias=True),
        # one shard of eight of a 12288 wide model
        dict(name="gate 12288 over 8", op="gate", back=False, dtype="bf16", rows=2048, width=12288, inner=6144, act="silu", bias=False),
        # the backward pass of a mid-size block, a microbatch that fills no tile
        dict(name="gate 2048 ragged back", op="gate", back=True, dtype="bf16", rows=1998, width=2048, inner=5504, act="silu", bias=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rotary", "attention", "attention", "gate"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "fp32"])
    if op == "gate":
        rows, width, inner = _log(rng, 1, 8192), 8 * _log(rng, 32, 1536), 8 * _log(rng, 32, 1024)
        if dtype == "fp32":
            rows, width, inner = min(rows, 1024), min(width, 2048), min(inner, 4096)
        return dict(op=op, back=rng.random() < 0.5, dtype=dtype, rows=rows, width=width, inner=inner,
                    act=rng.choice(["silu", "gelu_erf", "gelu_tanh", "sigmoid", "relu"]), bias=rng.random() < 0.5)
    dh, group = rng.choice([32, 64, 96, 128, 160]), rng.choice([1, 1, 2, 4, 5, 8])
    kv = rng.choice([1, 2, 3, 4, 8])
    heads, b = kv * group, rng.choice([1, 1, 2, 3, 4])
    if op == "rotary":
        s = _log(rng, 1, 16384)
        rot = rng.choice([dh, dh // 2])
        return dict(op=op, back=rng.random() < 0.5, dtype=dtype, s=s, b=b, heads=heads, kv=kv, dh=dh, rot=rot, pairs=rng.random() < 0.5,
                    scaling=rng.choice(["plain", "linear", "base", "ramp"]), places=rng.random() < 0.5)
    s = _log(rng, 1, 8192 if dtype == "bf16" else 512)
    if s > 2048:   # no dearer than the longest listed one
        b, heads, kv = 1, min(heads, 16) // kv * kv or kv, kv
    causal = rng.random() < 0.8
    docs = rng.choice([0, 0, max(1, s // 5), max(1, s // 2)])
    prefix = causal and rng.random() < 0.25
    window = 0 if prefix or rng.random() < 0.75 else max(1, s // 3)
    return dict(op=op, back=rng.random() < 0.6, dtype=dtype, s=s, b=b, heads=heads, kv=kv, dh=dh, cap=rng.choice([0.0, 0.0, 20.0, 50.0]),
                bias=rng.random() < 0.3, causal=causal, docs=docs, prefix=prefix, window=window)


def _documents(case, seed):
    """Document of every token [s, b] and the prefix length of every token's document; the last tokens of a sample may be padding (-1)."""
    r = np.random.RandomState(seed % (1 << 31))
    s, b = case["s"], case["b"]
    doc, prefix = np.zeros((s, b), np.int32), np.zeros((s, b), np.int32)
    for j in range(b):
        at, n = 0, 0
        while at < s:
            length = s if not case["docs"] else min(s - at, max(1, int(case["docs"] * r.uniform(0.2, 1.8))))
            doc[at:at + length, j] = n
            prefix[at:at + length, j] = r.randint(0, length + 1)
            at, n = at + length, n + 1
        if case["docs"]:
            doc[s - r.randint(0, max(1, s // 16)):, j] = -1
    return doc, prefix


def _visible_pairs(case):
    """Query/key pairs that see each other, of one head over all samples."""
    doc, prefix = _documents(case, 7)
    total = 0
    for j in range(case["b"]):
        d = doc[:, j]
        cuts = [0] + [i for i in range(1, case["s"]) if d[i] != d[i - 1]] + [case["s"]]
        for a, e in zip(cuts, cuts[1:]):
            if d[a] < 0:
                continue
            i = np.arange(a, e)
            w, p = case["window"], a + (prefix[a, j] if case["prefix"] else 0)
            lo = np.maximum(a, i - w + 1) if w else np.full_like(i, a)
            hi = np.maximum(i + 1, min(p, e)) if case["causal"] else (np.minimum(e, i + w) if w else np.full_like(i, e))
            total += int((hi - lo).sum())
    return total


class _State:
    pass


def _turns(case):
    """Turns per position of every pair, in 64 bits."""
    rot = case["rot"]
    base, factor, trained = 10000.0, 8.0, 4096.0
    if case["scaling"] == "base":
        base *= factor ** (rot / max(1, rot - 2))
    f = base ** (-2.0 * np.arange(rot // 2) / rot) / (2 * math.pi)
    if case["scaling"] == "linear":
        f = f / factor
    if case["scaling"] == "ramp":
        g = np.clip((trained * f - 1.0) / (32.0 - 1.0), 0.0, 1.0)
        f = f * (g + (1 - g) / factor)
    return f


def prepare(case, seed):
    st = _State()
    st.case = case
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    randn = lambda *shape, scale=1.0: (torch.randn(*shape, generator=g, device=DEV) * scale).to(dt)  # noqa: E731
    if case["op"] == "gate":
        rows, width, inner = case["rows"], case["width"], case["inner"]
        st.bias = randn(2 * inner, scale=0.1) if case["bias"] else None
        if case["back"]:
            st.dy, st.w2 = randn(rows, width), randn(inner, width, scale=0.02)
            st.z = randn(rows, 2 * inner)
            st.dz = torch.empty_like(st.z)
            st.dbias = torch.zeros(2 * inner, device=DEV) if case["bias"] else None
        else:
            st.u, st.w = randn(rows, width), randn(width, 2 * inner, scale=width ** -0.5)
            st.z, st.g = torch.empty(rows, 2 * inner, dtype=dt, device=DEV), torch.empty(rows, inner, dtype=dt, device=DEV)
        return st
    s, b, heads, kv, dh = (case[k] for k in ("s", "b", "heads", "kv", "dh"))
    row = (heads + 2 * kv) * dh
    st.qkv = randn(s, b, row)
    st.out = torch.empty_like(st.qkv)
    if case["op"] == "rotary":
        st.turns = torch.from_numpy(_turns(case)).to(DEV)
        # positions start again at boundaries of packed documents, some of them far into a long context
        st.positions = None
        if case["places"]:
            st.positions = torch.randint(0, 100000, (1, b), generator=g, device=DEV, dtype=torch.int32) + \
                torch.arange(s, device=DEV, dtype=torch.int32)[:, None] % max(1, s // 3)
        st.amplitude = 1.0 if case["scaling"] != "ramp" else 0.1 * math.log(8.0) + 1.0
        return st
    st.qkv[..., :heads * dh] *= 2   # scores of a trained model: sharper than at initialisation
    st.ctx, st.lse = torch.empty(s, b, heads * dh, dtype=dt, device=DEV), torch.empty(b, heads, s, device=DEV)
    st.dctx = randn(s, b, heads * dh)
    st.slopes = torch.from_numpy(2.0 ** (-8.0 * np.arange(1, heads + 1) / heads)).to(torch.float32).to(DEV) if case["bias"] else None
    doc, prefix = _documents(case, seed)
    st.doc = torch.from_numpy(doc).to(DEV) if case["docs"] else None
    st.prefix = torch.from_numpy(prefix).to(DEV) if case["prefix"] else None
    return st


# ---------------------------------------------------------------------------------------------- plain forms
def _plain_rotary(st):
    c = st.case
    s, b, heads, kv, dh, rot = (c[k] for k in ("s", "b", "heads", "kv", "dh", "rot"))
    place = st.positions if st.positions is not None else torch.arange(s, device=DEV)[:, None].expand(s, b)
    turn = place.to(torch.float64)[..., None] * st.turns
    angle = (turn - turn.floor()) * (2 * math.pi)
    cos, sin = (angle.cos() * st.amplitude).float()[:, :, None], (angle.sin() * st.amplitude).float()[:, :, None]
    if c["back"]:
        sin = -sin
    out = st.qkv.clone()
    x = out.view(s, b, heads + 2 * kv, dh)[:, :, :heads + kv, :rot]
    x = x.unflatten(-1, (rot // 2, 2)) if c["pairs"] else x.unflatten(-1, (2, rot // 2)).transpose(-1, -2)
    a, e = x[..., 0].float(), x[..., 1].float()
    x.copy_(torch.stack((a * cos - e * sin, a * sin + e * cos), -1))
    return dict(out=out)


def _plain_visible(st):
    """[b, s, s]: query sees key."""
    c = st.case
    i = torch.arange(c["s"], device=DEV)
    if st.doc is not None:
        d = st.doc.T
        run = torch.cat((torch.zeros_like(d[:, :1]), (d[:, 1:] != d[:, :-1]).int()), 1).cumsum(1)
        seen = (run[:, :, None] == run[:, None, :]) & (d >= 0)[:, :, None]
        first = (run[:, None, :] < run[:, :, None]).sum(-1)   # first token of the query's document
    else:
        seen = torch.ones(c["b"], c["s"], c["s"], dtype=torch.bool, device=DEV)
        first = torch.zeros(c["b"], c["s"], dtype=torch.int64, device=DEV)
    if c["causal"]:
        early = (i[None, :] <= i[:, None])[None]
        if st.prefix is not None:
            length = st.prefix.T.gather(1, first)   # as the document's first token has it
            early = early | (i[None, None, :] < (first + length)[:, :, None])
        seen = seen & early
    if c["window"]:
        seen = seen & ((i[:, None] - i[None, :]).abs() < c["window"])
    return seen


def _plain_attention(st):
    c = st.case
    s, b, heads, kv, dh = (c[k] for k in ("s", "b", "heads", "kv", "dh"))
    scale, group = dh ** -0.5, heads // kv
    x = st.qkv.float().view(s, b, heads + 2 * kv, dh).permute(1, 2, 0, 3)
    q = x[:, :heads].reshape(b, kv, group * s, dh)   # the heads of a group, one after the other
    k, v = x[:, heads:heads + kv].contiguous(), x[:, heads + kv:].contiguous()
    score = (torch.matmul(q, k.transpose(-1, -2).contiguous()) * scale).view(b, heads, s, s)
    steep = None
    if c["cap"]:
        t = torch.tanh(score / c["cap"])
        if c["back"]:
            steep = 1 - t * t
        score = c["cap"] * t
        del t
    if st.slopes is not None:
        i = torch.arange(s, device=DEV, dtype=torch.float32)
        score = score - st.slopes[:, None, None] * (i[:, None] - i[None, :]).abs()
    score.masked_fill_(~_plain_visible(st)[:, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    top = torch.where(top.isinf(), torch.zeros_like(top), top)
    p = torch.exp(score - top)
    del score
    total = p.sum(-1, keepdim=True)
    lse = torch.log(total) + top   # no key: log 0
    p = (p / torch.where(total == 0, torch.ones_like(total), total)).view(b, kv, group * s, s)
    ctx = torch.matmul(p, v)
    dt = st.qkv.dtype
    rows = lambda y, n: y.reshape(b, n, s, dh).permute(2, 0, 1, 3)  # noqa: E731
    out = dict(ctx=rows(ctx, heads).reshape(s, b, heads * dh).to(dt), lse=lse.view(b, heads, s))
    if not c["back"]:
        return out
    do = st.dctx.float().view(s, b, heads, dh).permute(1, 2, 0, 3).reshape(b, kv, group * s, dh)
    dv = torch.matmul(p.transpose(-1, -2).contiguous(), do)
    ds = torch.matmul(do, v.transpose(-1, -2).contiguous())
    ds -= (do * ctx).sum(-1, keepdim=True)
    ds *= p
    del p
    if steep is not None:
        ds *= steep.view(b, kv, group * s, s)
        del steep
    ds *= scale
    dq, dk = torch.matmul(ds, k), torch.matmul(ds.transpose(-1, -2).contiguous(), q)
    out["dqkv"] = torch.cat((rows(dq, heads), rows(dk, kv), rows(dv, kv)), 2).reshape(s, b, -1).to(dt)
    return out


def _plain_act(a, kind):
    """The activation and its derivative."""
    if kind == "relu":
        return a.clamp(min=0), (a > 0).float()
    if kind == "gelu_erf":
        cdf = 0.5 * (1 + torch.erf(a * math.sqrt(0.5)))
        return a * cdf, cdf + a * torch.exp(-0.5 * a * a) * (1 / math.sqrt(2 * math.pi))
    if kind == "gelu_tanh":
        k = math.sqrt(2 / math.pi)
        t = torch.tanh(k * (a + 0.044715 * a * a * a))
        return 0.5 * a * (1 + t), 0.5 * (1 + t) + 0.5 * a * (1 - t * t) * k * (1 + 3 * 0.044715 * a * a)
    s = 1 / (1 + torch.exp(-a))
    return (s, s * (1 - s)) if kind == "sigmoid" else (a * s, s * (1 + a * (1 - s)))


def _plain_gate(st):
    c = st.case
    inner = c["inner"]
    dt = st.z.dtype
    if not c["back"]:
        z = st.u.float() @ st.w.float()
        zb = z + st.bias.float() if st.bias is not None else z
        return dict(z=z.to(dt), g=(_plain_act(zb[:, :inner], c["act"])[0] * zb[:, inner:]).to(dt))
    dg = st.dy.float() @ st.w2.float().T
    zb = st.z.float() + st.bias.float() if st.bias is not None else st.z.float()
    f, df = _plain_act(zb[:, :inner], c["act"])
    dz = torch.cat((dg * df * zb[:, inner:], dg * f), 1)
    out = dict(dz=dz.to(dt))
    if st.bias is not None:
        out["dbias"] = dz.sum(0)
    return out


# ---------------------------------------------------------------------------------------------- the framework's kernels
def _at(t):
    return None if t is None else t.data_ptr()


def _workspace(st, size):
    if not hasattr(st, "ws"):
        st.ws = torch.empty(max(16, size), dtype=torch.uint8, device=DEV)
    return st.ws.data_ptr()


def _own_rotary(st, B):
    c = st.case
    call = B.ptdp_rotary_bwd if c["back"] else B.ptdp_rotary_fwd
    B.check(call(B.BF16 if c["dtype"] == "bf16" else B.F32, B.ROTARY_PAIRS if c["pairs"] else B.ROTARY_HALVES, _at(st.qkv), _at(st.positions),
                 _at(st.turns), _at(st.out), c["s"], c["b"], c["heads"], c["kv"], c["dh"], c["rot"], st.amplitude, B.stream_handle()), "rotary")
    return dict(out=st.out)


def _own_attention(st, B):
    c = st.case
    stream = B.stream_handle()
    cfg = B.make_span_cfg(c["s"], c["b"], c["heads"], c["kv"], c["dh"], B.BF16 if c["dtype"] == "bf16" else B.F32, cap=c["cap"])
    spans = None   # the causal mask alone needs none
    if not c["causal"] or c["window"] or st.doc is not None or st.prefix is not None:
        if not hasattr(st, "spans"):
            st.spans = torch.empty(B.ptdp_attn_spans_bytes(c["s"], c["b"]), dtype=torch.uint8, device=DEV)
        spans = _at(st.spans)
        B.check(B.ptdp_attn_spans(int(c["causal"]), c["window"], _at(st.doc), _at(st.prefix), spans, c["s"], c["b"], stream), "spans")
    cfg = C.byref(cfg)
    B.check(B.ptdp_attn_span_fwd(cfg, _at(st.qkv), spans, _at(st.slopes), _at(st.ctx), _at(st.lse), stream), "span_fwd")
    out = dict(ctx=st.ctx, lse=st.lse)
    if c["back"]:
        ws = _workspace(st, B.ptdp_attn_span_workspace_bytes(cfg))
        B.check(B.ptdp_attn_span_bwd(cfg, _at(st.qkv), spans, _at(st.slopes), _at(st.ctx), _at(st.lse), _at(st.dctx), _at(st.out), ws, stream),
                "span_bwd")
        out["dqkv"] = st.out
    return out


def _own_gate(st, B):
    c = st.case
    dtype, stream = B.BF16 if c["dtype"] == "bf16" else B.F32, B.stream_handle()
    act = dict(silu=B.GATE_SILU, gelu_erf=B.GATE_GELU_ERF, gelu_tanh=B.GATE_GELU_TANH, sigmoid=B.GATE_SIGMOID, relu=B.GATE_RELU)[c["act"]]
    size = c["rows"], c["width"], c["inner"]
    if not c["back"]:
        B.check(B.ptdp_gated_mlp_fwd(dtype, act, _at(st.u), _at(st.w), _at(st.bias), _at(st.z), _at(st.g), *size, stream), "gated_mlp_fwd")
        return dict(z=st.z, g=st.g)
    ws = _workspace(st, B.ptdp_gated_mlp_workspace_bytes(dtype, *size))
    if st.dbias is not None:
        st.dbias.zero_()   # gradients accumulate
    B.check(B.ptdp_gated_mlp_bwd(dtype, act, _at(st.dy), _at(st.w2), _at(st.z), _at(st.bias), _at(st.dz), _at(st.dbias), ws, *size, stream),
            "gated_mlp_bwd")
    return dict(dz=st.dz) if st.dbias is None else dict(dz=st.dz, dbias=st.dbias)


def run(st):
    if own:
        from paper_2104_04473_amd import binding as B
        return dict(rotary=_own_rotary, attention=_own_attention, gate=_own_gate)[st.case["op"]](st, B)
    return dict(rotary=_plain_rotary, attention=_plain_attention, gate=_plain_gate)[st.case["op"]](st)


def work(case):
    """Bytes: every input read once, every output written once.  FLOPs: the matrix products over visible pairs, the rotation's six per
    rotated element, a step's backward two and a half times its forward."""
    c = case
    e = 2 if c["dtype"] == "bf16" else 4
    if c["op"] == "gate":
        rows, width, inner = c["rows"], c["width"], c["inner"]
        if c["back"]:
            return dict(bytes=e * (rows * width + inner * width + 4 * rows * inner), flops=2.0 * rows * width * inner)
        return dict(bytes=e * (rows * width + 2 * inner * width + 3 * rows * inner), flops=4.0 * rows * width * inner)
    tokens, row = c["s"] * c["b"], (c["heads"] + 2 * c["kv"]) * c["dh"]
    if c["op"] == "rotary":
        return dict(bytes=2 * e * tokens * row + (4 * tokens if c["places"] else 0), flops=3.0 * tokens * (c["heads"] + c["kv"]) * c["rot"])
    ctx = tokens * c["heads"] * c["dh"]
    pairs = _visible_pairs(c) * c["heads"]
    if c["back"]:   # the forward's ctx is written, and read with dctx by the backward
        return dict(bytes=e * (3 * tokens * row + 3 * ctx), flops=14.0 * c["dh"] * pairs)
    return dict(bytes=e * (tokens * row + ctx), flops=4.0 * c["dh"] * pairs)


# ---------------------------------------------------------------------------------------------- in 64 bits, from the definitions
def _exact_rotary(st):
    """Pairs as complex numbers, multiplied by amplitude * exp(2 pi i position turns)."""
    c = st.case
    s, b, heads, kv, rot = (c[k] for k in ("s", "b", "heads", "kv", "rot"))
    place = torch.arange(s, device=DEV, dtype=torch.float64)[:, None].expand(s, b) if st.positions is None else st.positions.double()
    turn = torch.remainder(place[:, :, None, None] * st.turns, 1.0)
    z = torch.polar(torch.full_like(turn, st.amplitude), turn * (2 * math.pi))
    if c["back"]:
        z = z.conj()
    out = st.qkv.double().view(s, b, heads + 2 * kv, c["dh"]).clone()
    x = out[:, :, :heads + kv, :rot]
    if c["pairs"]:
        y = torch.view_as_real(torch.complex(x[..., 0::2].contiguous(), x[..., 1::2].contiguous()) * z).flatten(-2)
    else:
        h = torch.complex(x[..., :rot // 2].contiguous(), x[..., rot // 2:].contiguous()) * z
        y = torch.cat((h.real, h.imag), -1)
    out[:, :, :heads + kv, :rot] = y
    return dict(out=out.view(s, b, -1))


def _exact_spans(st):
    """First visible key and the one behind the last, [b][s], by walking the documents."""
    c = st.case
    s = c["s"]
    doc = st.doc.cpu().numpy() if st.doc is not None else np.zeros((s, c["b"]), np.int32)
    prefix = st.prefix.cpu().numpy() if st.prefix is not None else np.zeros((s, c["b"]), np.int32)
    lo, hi = np.zeros((c["b"], s), np.int64), np.zeros((c["b"], s), np.int64)
    for j in range(c["b"]):
        a = 0
        while a < s:
            e = a + 1
            while e < s and doc[e, j] == doc[a, j]:
                e += 1
            for i in range(a, e):
                if doc[a, j] < 0:
                    continue
                lo[j, i], hi[j, i] = a, e
                if c["causal"]:
                    hi[j, i] = max(i + 1, min(e, a + prefix[a, j]))
                if c["window"]:
                    lo[j, i], hi[j, i] = max(lo[j, i], i - c["window"] + 1), min(hi[j, i], i + c["window"])
            a = e
    return lo, hi


def _exact_attention(st):
    """Head by head, gradients by differentiation."""
    c = st.case
    s, b, heads, kv, dh = (c[k] for k in ("s", "b", "heads", "kv", "dh"))
    lo, hi = (torch.from_numpy(a).to(DEV) for a in _exact_spans(st))
    x = st.qkv.double().view(s, b, heads + 2 * kv, dh)
    grad = torch.zeros_like(x)
    ctx, lse = torch.zeros(s, b, heads, dh, dtype=torch.float64, device=DEV), torch.zeros(b, heads, s, dtype=torch.float64, device=DEV)
    i = torch.arange(s, device=DEV)
    for j in range(b):
        hidden = (i[None, :] < lo[j, :, None]) | (i[None, :] >= hi[j, :, None])
        empty = hidden.all(1)
        for h in range(heads):
            part = [x[:, j, n].clone().requires_grad_(c["back"]) for n in (h, heads + h // (heads // kv), heads + kv + h // (heads // kv))]
            score = part[0] @ part[1].T / math.sqrt(dh)
            if c["cap"]:
                score = c["cap"] * torch.tanh(score / c["cap"])
            if st.slopes is not None:
                score = score - st.slopes[h].double() * (i[:, None] - i[None, :]).abs()
            score = score.masked_fill(hidden, -math.inf)
            lse[j, h] = torch.logsumexp(score.detach(), 1)
            o = torch.softmax(score.masked_fill(empty[:, None], 0.0), 1).masked_fill(empty[:, None], 0.0) @ part[2]
            ctx[:, j, h] = o.detach()
            if c["back"]:
                for n, d in zip((h, heads + h // (heads // kv), heads + kv + h // (heads // kv)),
                                torch.autograd.grad(o, part, st.dctx[:, j, h * dh:(h + 1) * dh].double())):
                    grad[:, j, n] += d
    out = dict(ctx=ctx.view(s, b, -1), lse=lse)
    if c["back"]:
        out["dqkv"] = grad.view(s, b, -1)
    return out


def _exact_gate(st):
    c = st.case
    inner = c["inner"]
    act = dict(silu=torch.nn.functional.silu, gelu_erf=torch.nn.functional.gelu, sigmoid=torch.sigmoid, relu=torch.relu,
               gelu_tanh=lambda a: torch.nn.functional.gelu(a, approximate="tanh"))[c["act"]]
    z = (st.z.double() if c["back"] else st.u.double() @ st.w.double()).requires_grad_(c["back"])
    zb = z + (st.bias.double() if st.bias is not None else 0.0)
    g = act(zb[:, :inner]) * zb[:, inner:]
    if not c["back"]:
        return dict(z=z, g=g)
    dz, = torch.autograd.grad(g, z, st.dy.double() @ st.w2.double().T)
    return dict(dz=dz) if st.bias is None else dict(dz=dz, dbias=dz.sum(0))


def exact(case, seed):
    st = prepare(case, seed)
    return dict(rotary=_exact_rotary, attention=_exact_attention, gate=_exact_gate)[case["op"]](st)
