"""The gated projections of a feed-forward block and their gradient, against their definitions in 64 bits.

Bounds.  u is the unit round-off of the result's type (bf16 2^-8, fp16 2^-11).  A sum of c exact products in 32 bits is off by at most
c * 2^-23 times the sum of their magnitudes (2^-23 per addition also where an adder truncates).  The sigmoid of k is off by
r = 2^-20 + |k| 2^-21 of its value: exponential and reciprocal 2^-22 each, the exponent |k| by some units of 2^-24 of itself.  The
activation's slope is at most 1.13.  dgate and dup are rounded to 16 bits once before they are operands.
"""
import ctypes as C
import math

import pytest
import torch

import paper_1310_4645_b200 as rd
from test_norm import P, refused
from test_vocab import TINY, U, gen, ints, rand, strided, within

gpu = pytest.mark.gpu
HALF = [torch.bfloat16, torch.float16]
E4M3 = torch.float8_e4m3fn
ACTS = [rd.RD_SILU, rd.RD_GELU, rd.RD_RELU]


def activation(act, g):
    """(value, slope, bound of the value's error, bound of the slope's) in 64 bits."""
    if act == rd.RD_RELU:
        return g.clamp(min=0), (g > 0).double(), 0 * g, 0 * g
    c = 2 * math.sqrt(2 / math.pi)
    k, dk = (g, torch.ones_like(g)) if act == rd.RD_SILU else (c * (g + 0.044715 * g ** 3), c * (1 + 0.134145 * g * g))
    s = torch.sigmoid(k)
    r = 2.0 ** -20 + k.abs() * 2.0 ** -21
    return g * s, s + g * s * (1 - s) * dk, g.abs() * s * r + 2.0 ** -120, s * r + (g * dk).abs() * (s * r + 2.0 ** -23) + 2.0 ** -22


def project(x, w, scale=None):
    """A projection and the bound of its error."""
    y, err = x @ w.T, (x.abs() @ w.abs().T) * (x.shape[1] + 4) * 2.0 ** -23
    if scale is not None:
        y, err = y * scale, err * scale
        err = err + 2.0 ** -22 * y.abs()
    return y, err


def outside_untouched(view):
    """What lies between and behind the rows of a strided() tensor is still NaN."""
    base = view._base if view._base is not None else view
    kept = base.clone()
    kept.as_strided(view.shape, view.stride(), view.storage_offset()).fill_(math.nan)
    return bool(torch.isnan(kept).all())


def blank(rows, cols, dtype, pad=0, offset=0):
    return strided(torch.full((rows, cols), 7.0, dtype=dtype, device="cuda"), pad, offset)


SHAPES = [(1, 1, 1), (1, 64, 64), (1, 4096, 520), (1, 1000, 1001), (2, 33, 7000), (3, 40, 33), (7, 8, 16), (16, 512, 3000), (33, 72, 130), (100, 200, 20000), (128, 256, 300), (129, 64, 128),
          (200, 1000, 2730), (300, 520, 1000), (513, 129, 257), (64, 4096, 1111), (260, 2048, 64), (1000, 64, 2000), (130, 70, 30000), (2500, 264, 520)]


@gpu
@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("n, dim, width", SHAPES)
def test_gated(dtype, n, dim, width):
    std = 1.5 / math.sqrt(dim)
    x, wg, wu = rand(n, dim, seed=1, dtype=dtype), rand(width, dim, seed=2, dtype=dtype, std=std), rand(width, dim, seed=3, dtype=dtype, std=std)
    (g, eg), (u, eu) = project(x.double(), wg.double()), project(x.double(), wu.double())
    for k, act in enumerate(ACTS):
        v, _, ev, _ = activation(act, g)
        # aligned, rows with a stride, rows that nothing can address
        pad, offset = ((0, 0), (8, 0), (3, 1))[(k + n) % 3]
        put = lambda t: strided(t, pad, offset)
        out, gate, up = (blank(n, width, dtype, pad, offset) for _ in range(3))
        got = rd.rd_gated(put(x), put(wg), put(wu), act, out=out, gate=gate, up=up)
        assert got[0] is out and got[1] is gate and got[2] is up
        within(gate, g, eg + U[dtype] * (g.abs() + eg) + TINY[dtype])
        within(up, u, eu + U[dtype] * (u.abs() + eu) + TINY[dtype])
        bv = ev + 1.13 * eg
        bound = bv * (u.abs() + eu) + v.abs() * eu + 2.0 ** -23 * (v * u).abs()
        within(out, v * u, bound + U[dtype] * ((v * u).abs() + bound) + TINY[dtype])
        assert all(map(outside_untouched, (out, gate, up)))
        # the same bits wherever the operands lie, and whatever is kept
        o2, g2, u2 = rd.rd_gated(x, wg, wu, act)
        assert g2 is None and u2 is None and torch.equal(o2, out)
    assert rd.rd_block_status() == rd.RD_OK


@gpu
@pytest.mark.parametrize("n, dim, width", SHAPES)
def test_gated_8bit(n, dim, width):
    def eight(rows, seed):
        t = rand(rows, dim, seed=seed)
        scale = t.abs().amax(1) / 448
        return (t / scale[:, None]).to(E4M3), scale

    (x, sx), (wg, sg), (wu, su) = eight(n, 4), eight(width, 5), eight(width, 6)
    sg, su = sg / math.sqrt(dim), su / math.sqrt(dim)
    out_of = lambda s: sx.double()[:, None] * s.double()
    (g, eg), (u, eu) = project(x.float().double(), wg.float().double(), out_of(sg)), project(x.float().double(), wu.float().double(), out_of(su))
    for k, act in enumerate(ACTS):
        dtype = HALF[(k + n) % 2]
        v, _, ev, _ = activation(act, g)
        pad, offset = ((0, 0), (16, 0), (3, 1))[(k + n) % 3]

        def put(t):
            big = torch.zeros(t.shape[0] * (dim + pad) + offset, dtype=torch.uint8, device="cuda")
            view = big[offset:].view(t.shape[0], dim + pad)[:, :dim]
            view.copy_(t.view(torch.uint8))
            return view.view(E4M3)

        out, gate, up = (blank(n, width, dtype, pad, offset) for _ in range(3))
        rd.rd_gated(put(x), put(wg), put(wu), act, x_scale=sx, gate_scale=sg, up_scale=su, out_dtype=dtype, out=out, gate=gate, up=up)
        within(gate, g, eg + U[dtype] * (g.abs() + eg) + TINY[dtype])
        within(up, u, eu + U[dtype] * (u.abs() + eu) + TINY[dtype])
        bv = ev + 1.13 * eg
        bound = bv * (u.abs() + eu) + v.abs() * eu + 2.0 ** -23 * (v * u).abs()
        within(out, v * u, bound + U[dtype] * ((v * u).abs() + bound) + TINY[dtype])
        o2, _, _ = rd.rd_gated(x, wg, wu, act, x_scale=sx, gate_scale=sg, up_scale=su, out_dtype=dtype)
        assert torch.equal(o2, out)
    assert rd.rd_gated(x, wg, wu, x_scale=sx, gate_scale=sg, up_scale=su)[0].dtype == torch.bfloat16
    assert rd.rd_block_status() == rd.RD_OK


@gpu
@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("n", [1, 40, 300])
def test_gated_special_values(dtype, n):
    """An infinity or NaN stays in its row and in its column."""
    dim, width = 72, 150
    x, wg, wu = rand(n, dim, seed=7, dtype=dtype), rand(width, dim, seed=8, dtype=dtype), rand(width, dim, seed=9, dtype=dtype)
    clean = rd.rd_gated(x, wg, wu)[0]
    for where in ("x", "gate", "up"):
        for bad in (math.nan, math.inf):
            t = {"x": x.clone(), "gate": wg.clone(), "up": wu.clone()}
            t[where][n // 2 if where == "x" else 77, 5] = bad
            out = rd.rd_gated(t["x"], t["gate"], t["up"])[0]
            rest = torch.ones_like(clean, dtype=torch.bool)
            if where == "x":
                rest[n // 2] = False
            else:
                rest[:, 77] = False
            assert torch.equal(out[rest], clean[rest])
            assert not math.isnan(bad) or torch.isnan(out[~rest]).all()
    # far out: the activation is the line, or zero
    far = torch.zeros(n, 8, dtype=dtype, device="cuda")
    far[:, 0] = 200
    w = torch.zeros(4, 8, dtype=dtype, device="cuda")
    w[:, 0] = torch.tensor([1.0, -1.0, 0.5, 0.0])
    one = torch.zeros(4, 8, dtype=dtype, device="cuda")
    one[:, 0] = 1 / 200
    for act in ACTS:
        out, _, up = rd.rd_gated(far, w, one, act, keep=True)
        assert torch.allclose(out.float(), torch.tensor([200.0, 0.0, 100.0, 0.0], device="cuda") * up.float(), rtol=2 * U[dtype], atol=0)


def grad_reference(d, x, wg, wu, gate, up, act, dtype):
    v, slope, ev, es = activation(act, gate)
    dg, du = d * up * slope, d * v
    eg = (d * up).abs() * es + 2.0 ** -22 * dg.abs()
    eu = d.abs() * ev + 2.0 ** -22 * du.abs()
    eg, eu = eg + U[dtype] * (dg.abs() + eg) + TINY[dtype], eu + U[dtype] * (du.abs() + eu) + TINY[dtype]
    n, width = d.shape
    dx = dg @ wg + du @ wu
    ex = (eg @ wg.abs() + eu @ wu.abs()) + ((dg.abs() + eg) @ wg.abs() + (du.abs() + eu) @ wu.abs()) * (2 * width + 200) * 2.0 ** -23
    return ((dx, ex), *((t.T @ x, e.T @ x.abs() + (t.abs() + e).T @ x.abs() * (n + 4) * 2.0 ** -23) for t, e in ((dg, eg), (du, eu))))


@gpu
@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("n, dim, width", SHAPES)
def test_gated_grad(dtype, n, dim, width):
    std = 1.0 / math.sqrt(dim)
    x, wg, wu = rand(n, dim, seed=11, dtype=dtype), rand(width, dim, seed=12, dtype=dtype, std=std), rand(width, dim, seed=13, dtype=dtype, std=std)
    gate, up, d = (rand(n, width, seed=14 + k, dtype=dtype, std=s) for k, s in enumerate((1.5, 1.0, 1.0)))
    for k, act in enumerate(ACTS):
        want = grad_reference(*(t.double() for t in (d, x, wg, wu, gate, up)), act, dtype)
        pad, offset = ((0, 0), (8, 0), (3, 1))[(k + n) % 3]
        put = lambda t: strided(t, pad, offset)
        outs = [blank(r, dim, dtype, pad, offset) for r in (n, width, width)]
        got = rd.rd_gated_grad(put(d), put(x), put(wg), put(wu), put(gate), put(up), act, grad_x=outs[0], grad_gate_weight=outs[1], grad_up_weight=outs[2])
        assert all(a is b for a, b in zip(got, outs))
        for o, (w, e) in zip(outs, want):
            within(o, w, e + U[dtype] * (w.abs() + e) + TINY[dtype])
        assert all(map(outside_untouched, outs))
        again = rd.rd_gated_grad(d, x, wg, wu, gate, up, act)
        assert all(map(torch.equal, again, outs))
    x_alone = rd.rd_gated_grad(d, x, wg, wu, gate, up, act, want_weights=False)
    assert x_alone[1] is None and x_alone[2] is None and torch.equal(x_alone[0], outs[0])
    weights = rd.rd_gated_grad(d, x, wg, wu, gate, up, act, want_x=False)
    assert weights[0] is None and torch.equal(weights[1], outs[1]) and torch.equal(weights[2], outs[2])
    into = torch.empty_like(wu)
    up_alone = rd.rd_gated_grad(d, x, wg, wu, gate, up, act, want_x=False, want_weights=False, grad_up_weight=into)
    assert up_alone[0] is None and up_alone[1] is None and torch.equal(into, outs[2])
    assert rd.rd_block_status() == rd.RD_OK


@gpu
def test_gated_no_rows_and_broadcast_rows():
    x, wg, wu = rand(5, 40, seed=20, dtype=torch.bfloat16), rand(24, 40, seed=21, dtype=torch.bfloat16), rand(24, 40, seed=22, dtype=torch.bfloat16)
    out, gate, up = rd.rd_gated(x[:0], wg, wu, keep=True)
    assert out.shape == gate.shape == up.shape == (0, 24)
    gx, gg, gu = rd.rd_gated_grad(out, x[:0], wg, wu, gate, up)
    assert gx.shape == (0, 40) and not gg.any() and not gu.any()
    one = x[:1].expand(200, 40)
    out, gate, up = rd.rd_gated(one, wg, wu, keep=True)
    same, _, _ = rd.rd_gated(one.contiguous(), wg, wu)
    assert torch.equal(out, same)
    d = rand(1, 24, seed=23, dtype=torch.bfloat16).expand(200, 24)
    for a, b in zip(rd.rd_gated_grad(d, one, wg, wu, gate, up), rd.rd_gated_grad(d.contiguous(), one.contiguous(), wg, wu, gate, up)):
        assert torch.equal(a, b)


@gpu
@pytest.mark.parametrize("act", ACTS)
def test_gated_grad_is_the_derivative(act):
    """Difference quotients of <d, out> in 64 bits, of the function that the forward pass computes, against the gradient."""
    n, dim, width, dtype = 6, 24, 20, torch.float16
    x, wg, wu, d = rand(n, dim, seed=30, dtype=dtype), rand(width, dim, seed=31, dtype=dtype, std=0.2), rand(width, dim, seed=32, dtype=dtype, std=0.2), rand(n, width, seed=33, dtype=dtype)
    out, gate, up = rd.rd_gated(x, wg, wu, act, keep=True)
    grads = rd.rd_gated_grad(d, x, wg, wu, gate, up, act)

    def value(x, wg, wu):
        return (d.double() * activation(act, x @ wg.T)[0] * (x @ wu.T)).sum().item()

    assert abs(value(x.double(), wg.double(), wu.double()) - (d.double() * out.double()).sum().item()) <= 2 * U[dtype] * (d.double() * out.double()).abs().sum().item()
    h = 1e-5
    for which, g in enumerate(grads):
        for i, j in ((0, 0), (5, 23), (3, 11)):
            t = [[v.double().clone() for v in (x, wg, wu)] for _ in range(2)]
            t[0][which][i, j] += h
            t[1][which][i, j] -= h
            quotient = (value(*t[0]) - value(*t[1])) / (2 * h)
            # kept gate and up, dgate, dup and the result are rounded to 16 bits: four roundings of terms whose magnitudes add up to
            # at most this; near 0 relu's slope is not rounded but jumps, which these places do not meet
            size = {0: (d.abs().double() @ (wg.abs() + wu.abs()).double() * 4).max(), 1: (d.abs().double().T @ x.abs().double() * 4).max(), 2: (d.abs().double().T @ x.abs().double() * 4).max()}[which].item()
            assert abs(quotient - g[i, j].item()) <= 4 * U[dtype] * size


@gpu
@pytest.mark.parametrize("n", [1, 50, 400])
def test_gated_streams_and_graphs(n):
    """On a stream of its own, on two at once, and two recordings played again on other inputs, with the bits of the plain calls."""
    dim, width, dtype = 136, 700, torch.bfloat16
    sets = [[rand(n, dim, seed=40 + 4 * k, dtype=dtype), rand(width, dim, seed=41 + 4 * k, dtype=dtype), rand(width, dim, seed=42 + 4 * k, dtype=dtype),
             rand(n, width, seed=43 + 4 * k, dtype=dtype)] for k in range(2)]

    def passes(x, wg, wu, d, stream=None):
        out, gate, up = rd.rd_gated(x, wg, wu, keep=True, stream=stream)
        return (out, gate, up, *rd.rd_gated_grad(d, x, wg, wu, gate, up, stream=stream))

    want = [passes(*s) for s in sets]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = [[passes(*s, stream=st) for s, st in zip(sets, streams)] for _ in range(3)]
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for turn in got for g, w in zip(turn, want) for a, b in zip(g, w))
    inputs = [t.clone() for t in sets[0]]
    graphs, results = [torch.cuda.CUDAGraph() for _ in range(2)], []
    for graph in graphs:
        with torch.cuda.graph(graph):
            results.append(passes(*inputs))
    for s, w in zip(sets, want):
        for a, b in zip(inputs, s):
            a.copy_(b)
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for r in results for a, b in zip(r, w))
    assert rd.rd_block_status() == rd.RD_OK


# ------------------------------------------------------------------------------------------------ refusals


GATED = dict(x=P, xs=8, wg=2 * P, wgs=8, wu=3 * P, wus=8, sx=None, sg=None, su=None, n=4, dim=8, width=16, dtype=rd.RD_BF16, act=rd.RD_SILU)
BAD_GATED = [dict(x=None), dict(wg=None), dict(wu=None), dict(x=P + 1), dict(wg=2 * P + 1), dict(wu=3 * P + 1), dict(xs=7), dict(wgs=7), dict(wus=7), dict(wgs=0), dict(dim=0), dict(width=0),
             dict(dim=65537, xs=65537, wgs=65537, wus=65537), dict(dtype=9), dict(act=3), dict(act=-1), dict(sx=4 * P), dict(sg=4 * P), dict(su=4 * P)]
UNSUPPORTED_GATED = [dict(dtype=rd.RD_FP32), dict(dtype=rd.RD_INT32), dict(n=1 << 31), dict(width=(1 << 20) + 1)]


def test_gated_refusals():
    L, need = rd.lib(), C.c_size_t(1)
    odd = {**GATED, "x": P + 2}
    assert L.rd_gated_workspace(C.byref(rd.rd_gated_t(*GATED.values())), C.byref(need)) == rd.RD_OK and need.value == 0
    assert L.rd_gated_workspace(C.byref(rd.rd_gated_t(*odd.values())), C.byref(need)) == rd.RD_OK and need.value > 0
    assert L.rd_gated_workspace(None, C.byref(need)) == rd.RD_ERR_INVALID_ARG
    assert L.rd_gated_workspace(C.byref(rd.rd_gated_t(*GATED.values())), None) == rd.RD_ERR_INVALID_ARG

    def call(out, os, ot, gate, gs, up, us, ws, size, **kw):
        return L.rd_gated(C.byref(rd.rd_gated_t(*kw.values())), out, os, ot, gate, gs, up, us, ws, size, None)

    good = dict(out=8 * P, os=16, ot=rd.RD_BF16, gate=9 * P, gs=16, up=10 * P, us=16, ws=None, size=0, **GATED)
    eight = dict(dtype=rd.RD_E4M3, sx=11 * P, sg=12 * P, su=13 * P)
    refused(call, good, BAD_GATED + [dict(out=None), dict(out=8 * P + 1), dict(gate=9 * P + 1), dict(up=10 * P + 1), dict(os=15), dict(gs=15), dict(us=15), dict(os=0), dict(ot=9),
                                     dict(out=P), dict(out=2 * P), dict(gate=3 * P), dict(up=8 * P), dict(up=9 * P + 2), dict(x=P + 2, ws=None, size=need.value),
                                     dict(x=P + 2, ws=16 * P + 8, size=need.value), dict(x=P + 2, ws=8 * P, size=need.value),
                                     {**eight, "sx": None}, {**eight, "sg": None}, {**eight, "su": None}, {**eight, "sx": 11 * P + 2}, {**eight, "out": 12 * P}],
            UNSUPPORTED_GATED + [dict(ot=rd.RD_FP16), dict(ot=rd.RD_FP32), {**eight, "ot": rd.RD_FP32}, {**eight, "ot": rd.RD_E4M3}])
    assert call(**{**good, "x": P + 2, "ws": 16 * P, "size": need.value - 1}) == rd.RD_ERR_TOO_SMALL
    assert call(**{**good, "n": 0, "x": None, "out": None}) == rd.RD_OK
    assert L.rd_block_status(None) == rd.RD_ERR_INVALID_ARG


def test_gated_grad_refusals():
    L, need = rd.lib(), C.c_size_t()
    assert L.rd_gated_grad_workspace(C.byref(rd.rd_gated_t(*GATED.values())), 1, C.byref(need)) == rd.RD_OK and need.value > 0
    assert L.rd_gated_grad_workspace(C.byref(rd.rd_gated_t(*GATED.values())), 1, None) == rd.RD_ERR_INVALID_ARG
    eight = dict(dtype=rd.RD_E4M3, sx=30 * P, sg=31 * P, su=32 * P)
    assert L.rd_gated_grad_workspace(C.byref(rd.rd_gated_t(*{**GATED, **eight}.values())), 1, C.byref(C.c_size_t())) == rd.RD_ERR_UNSUPPORTED

    def call(d, ds, gate, gs, up, us, gx, gxs, gg, ggs, gu, gus, ws, size, **kw):
        return L.rd_gated_grad(C.byref(rd.rd_gated_t(*kw.values())), d, ds, gate, gs, up, us, gx, gxs, gg, ggs, gu, gus, ws, size, None)

    good = dict(d=8 * P, ds=16, gate=9 * P, gs=16, up=10 * P, us=16, gx=11 * P, gxs=8, gg=12 * P, ggs=8, gu=13 * P, gus=8, ws=16 * P, size=need.value, **GATED)
    refused(call, good, BAD_GATED + [dict(gx=None, gg=None, gu=None), dict(d=None), dict(gate=None), dict(up=None), dict(d=8 * P + 1), dict(gate=9 * P + 1), dict(up=10 * P + 1),
                                     dict(gx=11 * P + 1), dict(gg=12 * P + 1), dict(gu=13 * P + 1), dict(ds=15), dict(gs=15), dict(us=15), dict(gxs=7), dict(ggs=7), dict(gus=7),
                                     dict(gxs=0), dict(ws=None), dict(ws=16 * P + 8), dict(gx=P), dict(gg=2 * P), dict(gu=3 * P), dict(gx=8 * P), dict(gg=9 * P), dict(gu=12 * P),
                                     dict(ws=10 * P), dict(ws=12 * P)],
            UNSUPPORTED_GATED + [eight])
    assert call(**{**good, "size": need.value - 1}) == rd.RD_ERR_TOO_SMALL
    assert call(**{**good, "n": 0, "x": None, "d": None, "gate": None, "up": None, "gg": None, "gu": None}) == rd.RD_OK


@gpu
def test_gated_binding_refusals():
    x, w = torch.zeros(4, 8, device="cuda").half(), torch.zeros(16, 8, device="cuda").half()
    d, s = torch.zeros(4, 16, device="cuda").half(), torch.ones(4, device="cuda")
    for f in (lambda: rd.rd_gated(x.cpu(), w, w), lambda: rd.rd_gated(x, w.cpu(), w), lambda: rd.rd_gated(x, w, w[:15]), lambda: rd.rd_gated(x, w, w.bfloat16()), lambda: rd.rd_gated(x, w[:, :7], w),
              lambda: rd.rd_gated(x[0], w, w), lambda: rd.rd_gated(x.T, w, w), lambda: rd.rd_gated(x, w, w, out=d[:3]), lambda: rd.rd_gated(x, w, w, gate=d.float()),
              lambda: rd.rd_gated(x, w, w, out_dtype=16), lambda: rd.rd_gated(x, w, w, x_scale=s.double()), lambda: rd.rd_gated(x, w, w, x_scale=s[:3]),
              lambda: rd.rd_gated_grad(d[:3], x, w, w, d, d), lambda: rd.rd_gated_grad(d, x, w, w, d, d.float()), lambda: rd.rd_gated_grad(d, x, w, w, d, d, grad_x=w),
              lambda: rd.rd_gated_grad(d, x, w, w, d, d, grad_gate_weight=x), lambda: rd.rd_gated_grad(d, x, w, w, d, d, workspace=torch.zeros(8))):
        with pytest.raises(ValueError):
            f()
    e = x.to(E4M3), w.to(E4M3)
    for f, code in ((lambda: rd.rd_gated(x.float(), w.float(), w.float()), rd.RD_ERR_UNSUPPORTED), (lambda: rd.rd_gated(x, w, w, 5), rd.RD_ERR_INVALID_ARG),
                    (lambda: rd.rd_gated(e[0], e[1], e[1]), rd.RD_ERR_INVALID_ARG), (lambda: rd.rd_gated(x, w, w, x_scale=s), rd.RD_ERR_INVALID_ARG),
                    (lambda: rd.rd_gated(x, w, w, out_dtype=torch.bfloat16), rd.RD_ERR_UNSUPPORTED),
                    (lambda: rd.rd_gated_grad(d, x, w, w, d, d, workspace=torch.zeros(255, device="cuda")), rd.RD_ERR_TOO_SMALL)):
        with pytest.raises(rd.RdError) as err:
            f()
        assert err.value.status == code
