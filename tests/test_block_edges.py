"""The block operators at the edges of what their documentation allows: broadcast operands, threads, matrices of more than 2^31 values."""
import threading

import pytest
import torch

import paper_1310_4645_b200 as rd
from test_gated import ACTS, HALF, activation, blank, grad_reference, outside_untouched, project
from test_norm import BF16, E, E4M3, FP32, kept
from test_vocab import TINY, U, gen, rand, strided, within

gpu = pytest.mark.gpu


@gpu
@pytest.mark.parametrize("dim", [64, 1000, 1001, 4096, 9000])
def test_norm_of_broadcast_rows(dim):
    """One row for all as x, residual or a gradient; x that is its own residual."""
    n = 70
    x, one, weight = rand(n, dim, seed=1, dtype=BF16), rand(1, dim, seed=2, dtype=BF16), rand(1, dim, seed=3)[0]
    same = lambda a, b: all((p is None and q is None) or torch.equal(p, q) for p, q in zip(a, b))
    wide = one.expand(n, dim)
    assert same(rd.rd_norm(wide, weight, x, drop=0.3, seed=4), rd.rd_norm(wide.contiguous(), weight, x, drop=0.3, seed=4))
    assert same(rd.rd_norm(x, weight, wide, out_dtype=E4M3), rd.rd_norm(x, weight, wide.contiguous(), out_dtype=E4M3))
    assert same(rd.rd_norm(x, weight, x), rd.rd_norm(x, weight, x.clone()))
    rstd = torch.rand(n, generator=gen(5), device="cuda")
    assert same(rd.rd_norm_grad(wide, x, weight, rstd, wide), rd.rd_norm_grad(wide.contiguous(), x, weight, rstd, wide.contiguous()))
    assert same(rd.rd_norm_grad(x, wide, weight, rstd, x, drop=0.2, seed=6), rd.rd_norm_grad(x, wide.contiguous(), weight, rstd, x.clone(), drop=0.2, seed=6))
    # in place of an input that is the other one, too
    t = x.clone()
    out, total, _, _ = rd.rd_norm(t, weight, t, total=t)
    assert total is t and same((out, total), rd.rd_norm(x, weight, x)[:2])


@gpu
def test_block_operators_from_threads():
    """Four threads with streams of their own, each with other inputs, against one thread's results."""
    n, dim, width = 150, 264, 520

    def inputs(k):
        return [rand(n, dim, seed=10 * k + 1, dtype=BF16), rand(n, dim, seed=10 * k + 2, dtype=BF16), rand(1, dim, seed=10 * k + 3)[0], rand(width, dim, seed=10 * k + 4, dtype=BF16),
                rand(width, dim, seed=10 * k + 5, dtype=BF16), rand(n, width, seed=10 * k + 6, dtype=BF16)]

    def passes(x, residual, weight, wg, wu, d, stream=None):
        out, total, rstd, _ = rd.rd_norm(x, weight, residual, drop=0.1, seed=9, stream=stream)
        act, gate, up = rd.rd_gated(out, wg, wu, keep=True, stream=stream)
        grads = rd.rd_gated_grad(d, out, wg, wu, gate, up, stream=stream)
        return (out, total, rstd, act, gate, up, *grads, *rd.rd_norm_grad(grads[0], total, weight, rstd, residual, drop=0.1, seed=9, stream=stream))

    sets = [inputs(k) for k in range(4)]
    want = [passes(*s) for s in sets]
    torch.cuda.synchronize()
    wrong = []

    def work(k):
        stream = torch.cuda.Stream()
        for _ in range(20):
            got = passes(*sets[k], stream=stream)
            stream.synchronize()
            if not all(map(torch.equal, got, want[k])):
                wrong.append(k)

    threads = [threading.Thread(target=work, args=(k,)) for k in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong and rd.rd_block_status() == rd.RD_OK


@gpu
@pytest.mark.parametrize("dim", [16384, 16381])
def test_norm_of_more_than_two_to_the_31_values(dim):
    n = (1 << 31) // dim + 9
    x = torch.empty(n, dim, dtype=BF16, device="cuda").normal_(generator=gen(20))
    weight = 1 + rand(1, dim, seed=21, std=0.2)[0]
    rows = torch.tensor([0, 1, n // 2, n - 2, n - 1], device="cuda")
    mask = torch.cat([kept(1, dim, 0.25, 22, 23, 7 + int(r)) for r in rows])
    s = x[rows].double() * mask
    want = s * (s.square().mean(1, keepdim=True) + 1e-6).rsqrt() * weight.double()
    dropped = rd.rd_dropout(x, 0.25, 22, 23, first_row=7)
    within(dropped[rows], s, (U[BF16] + E) * s.abs() + TINY[BF16])
    del dropped
    # a row's sum adds up fewer than 64 terms on any value's way; products, root and rounding
    bound = (U[BF16] + 80 * E) * want.abs() + TINY[BF16]
    out, total, rstd, _ = rd.rd_norm(x, weight, drop=0.25, seed=22, offset=23, first_row=7)
    within(out[rows], want, bound)
    del out
    gx, gr, gw = rd.rd_norm_grad(x, total, weight, rstd, drop=0.25, seed=22, offset=23, first_row=7, want_weight=False, grad_residual=total)
    assert gr is total
    u, r = x[rows].double() * weight.double(), rstd[rows].double()[:, None]
    # total was rounded to 16 bits; what the gradient read is that
    t = s.to(BF16).double()
    dot = (u * t).mean(1, keepdim=True)
    grad = r * (u - t * r * r * dot)
    size = r * (u.abs() + t.abs() * r * r * (u * t).abs().mean(1, keepdim=True))
    # s rounded to 16 bits here may be the neighbour of the kernel's: as much as a rounding of it again
    within(gx[rows], grad * mask, (2 * U[BF16] * size + U[BF16] * grad.abs()) * mask + TINY[BF16])


@gpu
def test_gated_of_more_than_two_to_the_31_values():
    n, dim, width = 180001, 64, 12000
    x, wg, wu = rand(n, dim, seed=30, dtype=BF16), rand(width, dim, seed=31, dtype=BF16, std=0.15), rand(width, dim, seed=32, dtype=BF16, std=0.15)
    out, gate, up = rd.rd_gated(x, wg, wu, keep=True)
    rows = torch.tensor([0, 1, n // 2, n - 2, n - 1], device="cuda")
    (g, eg), (u, eu) = project(x[rows].double(), wg.double()), project(x[rows].double(), wu.double())
    v, _, ev, _ = activation(rd.RD_SILU, g)
    bound = (ev + 1.13 * eg) * (u.abs() + eu) + v.abs() * eu + 2.0 ** -23 * (v * u).abs()
    within(out[rows], v * u, bound + U[BF16] * ((v * u).abs() + bound) + TINY[BF16])
    within(up[rows], u, eu + U[BF16] * (u.abs() + eu) + TINY[BF16])
    # gradients: only the last rows have any, so that the weights' are theirs
    out.zero_()
    out[rows[-2:]] = rand(2, width, seed=33, dtype=BF16)
    gx, gg, gu = rd.rd_gated_grad(out, x, wg, wu, gate, up)
    few = [t[rows[-2:]].contiguous() for t in (out, x, gate, up)]
    sx, sg, su = rd.rd_gated_grad(few[0], few[1], wg, wu, few[2], few[3])
    assert not gx[:-2].any()
    # the same products, added up in other parts: each sum within 2 * width (2) terms' roundings of the magnitudes
    assert (gx[-2:].double() - sx.double()).norm() <= 2 * U[BF16] * sx.double().norm()
    assert (gg.double() - sg.double()).norm() <= 2 * U[BF16] * sg.double().norm() and (gu.double() - su.double()).norm() <= 2 * U[BF16] * su.double().norm()
    assert rd.rd_block_status() == rd.RD_OK


@gpu
@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("n, dim, width", [(300, 40, 24), (1924, 64, 256), (1025, 1, 1), (4046, 192, 128), (3001, 130, 77), (6550, 256, 1003), (8170, 128, 2048), (2000, 24, 4100), (20000, 65, 129)])
def test_gated_grad_of_few_columns(dtype, n, dim, width):
    """Few tiles of the weights' gradients, and many rows that each is a sum over."""
    x, wg, wu = rand(n, dim, seed=61, dtype=dtype), rand(width, dim, seed=62, dtype=dtype, std=dim ** -0.5), rand(width, dim, seed=63, dtype=dtype, std=dim ** -0.5)
    gate, up, d = (rand(n, width, seed=64 + k, dtype=dtype) for k in range(3))
    act = ACTS[(n + width) % 3]
    want = grad_reference(*(t.double() for t in (d, x, wg, wu, gate, up)), act, dtype)
    first = None
    for pad, offset in ((0, 0), (8, 0), (2, 0), (2, 2), (3, 1)):
        put = lambda t: strided(t, pad, offset)
        outs = [blank(r, dim, dtype, pad, offset) for r in (n, width, width)]
        rd.rd_gated_grad(put(d), put(x), put(wg), put(wu), put(gate), put(up), act, grad_x=outs[0], grad_gate_weight=outs[1], grad_up_weight=outs[2])
        if first is None:
            first = outs
            for o, (w, e) in zip(outs, want):
                within(o, w, e + U[dtype] * (w.abs() + e) + TINY[dtype])
        assert all(map(torch.equal, outs, first)) and all(map(outside_untouched, outs))
    # what is wanted does not change the bits
    args = (d, x, wg, wu, gate, up, act)
    assert torch.equal(rd.rd_gated_grad(*args, want_weights=False)[0], first[0])
    assert all(map(torch.equal, rd.rd_gated_grad(*args, want_x=False)[1:], first[1:]))
    for k, name in ((1, "grad_gate_weight"), (2, "grad_up_weight")):
        for want_x in (False, True):
            into = torch.empty_like(wg)
            rd.rd_gated_grad(*args, want_x=want_x, want_weights=False, **{name: into})
            assert torch.equal(into, first[k])
    # recorded, and played again on other rows
    graph, inputs = torch.cuda.CUDAGraph(), [t.clone() for t in args[:-1]]
    with torch.cuda.graph(graph):
        got = rd.rd_gated_grad(*inputs, act)
    inputs[0].copy_(d.flip(0)), inputs[1].copy_(x.flip(0)), inputs[4].copy_(gate.flip(0)), inputs[5].copy_(up.flip(0))
    graph.replay()
    assert torch.equal(got[0], first[0].flip(0))
    assert all(map(torch.equal, got, rd.rd_gated_grad(*inputs, act)))
    assert rd.rd_block_status() == rd.RD_OK
