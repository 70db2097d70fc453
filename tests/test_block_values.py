"""Values at which the block operators are easily wrong: scales whose product leaves fp32's range, NaN and infinities
before 8 bits and in gradients, the range of fp16."""
import pytest
import torch

import paper_1310_4645_b200 as rd
from test_gated import E4M3, HALF, activation, grad_reference, project
from test_norm import BF16
from test_vocab import TINY, U, gen, rand, within

gpu = pytest.mark.gpu


@gpu
@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("n", [3, 200])
@pytest.mark.parametrize("x_power, w_power", [(-85, -62), (-60, -90), (-70, -66), (70, 75), (-100, 90), (100, -90)])
def test_gated_8bit_scales_one_after_the_other(dtype, n, x_power, w_power):
    """gate and up are products times the row's scale, times the column's: right wherever that order is, although the scales' own product
    may be too small or too large for fp32.  (Large powers: a few products are small enough for the result to fit, others are infinite.)"""
    dim, width = 1024, 72
    x, wg, wu = ((rand(r, dim, seed=k) * 100).to(E4M3) for k, r in ((1, n), (2, width), (3, width)))
    if x_power + w_power > 0:
        # products of single values, the smallest of which are subnormal numbers' squares
        x, wg, wu = ((t.float().sign() * 2.0 ** -9 * (torch.arange(dim, device="cuda") == 7)).to(E4M3) for t in (x, wg, wu))
    some = lambda r, seed: 1 + torch.rand(r, generator=gen(seed), device="cuda")
    sx, sg, su = (some(r, k) * 2.0 ** p for r, k, p in ((n, 4, x_power), (width, 5, w_power), (width, 6, w_power)))
    out, gate, up = rd.rd_gated(x, wg, wu, x_scale=sx, gate_scale=sg, up_scale=su, out_dtype=dtype, keep=True)
    most = torch.finfo(dtype).max
    for got, w, s in ((gate, wg, sg), (up, wu, su)):
        y, err = project(x.float().double(), w.float().double())
        # a product with a scale that is a subnormal number is off by half of their spacing, times the other scale
        y, err = y * sx.double()[:, None] * s.double(), (err * sx.double()[:, None] + 2.0 ** -150) * s.double()
        err = err + 2.0 ** -22 * y.abs() + 2.0 ** -150
        bound = err + U[dtype] * (y.abs() + err) + TINY[dtype]
        fits = y.abs() + bound < most
        zero = torch.zeros_like(y)
        within(torch.where(fits, got.double(), zero), torch.where(fits, y, zero), torch.where(fits, bound, zero))
        assert (got.double().abs()[y.abs() - bound > most * (1 + U[dtype])] == torch.inf).all()

@gpu
@pytest.mark.parametrize("dim", [64, 120, 256, 2000, 2001, 4096, 9000])
@pytest.mark.parametrize("dtype", [torch.float32, BF16])
def test_norm_8bit_with_a_nan(dtype, dim):
    """A NaN anywhere in a row's values, also one that the weight brings, is in the row's scale and in all of its 8-bit values."""
    x, weight = rand(5, dim, seed=1, dtype=dtype), 1 + rand(1, dim, seed=2, std=0.2)[0]
    clean, _, _, scale = rd.rd_norm(x, weight, x, out_dtype=E4M3)
    for bad in (torch.nan, torch.inf):
        for at in (0, dim // 2, dim - 1):
            y = x.clone()
            y[3, at] = bad
            q, _, _, s = rd.rd_norm(y, weight, x, out_dtype=E4M3)
            rest = torch.arange(5, device="cuda") != 3
            # an infinity times the reciprocal root 0 of its row
            assert torch.isnan(s[3]) and torch.isnan(q[3].float()).all()
            assert torch.equal(s[rest], scale[rest]) and torch.equal(q[rest].float(), clean[rest].float())
            w = weight.clone()
            w[at] = torch.nan
            q, _, _, s = rd.rd_norm(x, w, x, out_dtype=E4M3)
            assert torch.isnan(s).all() and torch.isnan(q.float()).all()
            # an infinite weight: the largest value is infinite, and times a zero NaN
            w[at] = torch.inf
            z = x.clone()
            z[2, at] = 0
            q, _, _, s = rd.rd_norm(z, w, z, out_dtype=E4M3)
            rest = torch.arange(5, device="cuda") != 2
            assert torch.isnan(s[2]) and torch.isnan(q[2].float()).all() and (s[rest] == torch.inf).all()
            assert torch.isnan(q[rest, at].float()).all() and not q[rest][:, torch.arange(dim, device="cuda") != at].float().any()


@gpu
@pytest.mark.parametrize("dim", [96, 2000, 4095])
def test_norm_8bit_of_zeros_without_eps(dim):
    """0 / 0, as without 8 bits; with an eps the scale is 0."""
    x, weight = torch.zeros(3, dim, device="cuda"), torch.ones(dim, device="cuda")
    q, _, rstd, scale = rd.rd_norm(x, weight, eps=0.0, out_dtype=E4M3)
    assert torch.isinf(rstd).all() and torch.isnan(scale).all() and torch.isnan(q.float()).all()
    q, _, _, scale = rd.rd_norm(x, weight, eps=2.0 ** -126, out_dtype=E4M3)
    assert not scale.any() and not q.float().any()


def limits(act, g):
    """(value, slope) as the gradient takes them at infinities: the slope's limit, and a value that is a product with a factor of 0."""
    value, slope, _, _ = activation(act, g)
    if act != rd.RD_RELU:
        value = torch.where(g == torch.inf, torch.inf, torch.where(g == -torch.inf, torch.nan, value))
        slope = torch.where(g == torch.inf, 1.0, torch.where(g == -torch.inf, 0.0, slope))
    return value, slope


@gpu
@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("n, dim, width", [(1, 24, 16), (40, 72, 150), (300, 136, 77), (2000, 64, 128)])
def test_gated_grad_special_values(dtype, n, dim, width):
    """An infinity or NaN in one place comes out where the formulas have it, and nowhere else."""
    i, j, k = n // 2, width // 3, dim - 1
    names = ("d", "x", "wg", "wu", "gate", "up")
    clean = dict(zip(names, (rand(*s, seed=10 + m, dtype=dtype) for m, s in enumerate(((n, width), (n, dim), (width, dim), (width, dim), (n, width), (n, width))))))
    for act in (rd.RD_SILU, rd.RD_GELU, rd.RD_RELU):
        want = rd.rd_gated_grad(*clean.values(), act)
        for name in names:
            for bad in (torch.nan, torch.inf, -torch.inf):
                t = {m: v.clone() for m, v in clean.items()}
                t[name][{"d": (i, j), "gate": (i, j), "up": (i, j), "x": (i, k), "wg": (j, k), "wu": (j, k)}[name]] = bad
                got = rd.rd_gated_grad(*t.values(), act)
                # where the result may differ at all
                touched = [torch.zeros_like(w, dtype=torch.bool) for w in want]
                if name in ("d", "gate", "up"):
                    touched[0][i] = touched[1][j] = touched[2][j] = True
                elif name == "x":
                    touched[1][:, k] = touched[2][:, k] = True
                else:
                    touched[0][:, k] = True
                if name == "up":
                    touched[2][:] = False
                assert all(torch.equal(g[~m], w[~m]) for g, w, m in zip(got, want, touched))
                s = {m: v.double() for m, v in t.items()}
                value, slope = limits(act, s["gate"])
                dg, du = s["d"] * s["up"] * slope, s["d"] * value
                for g, r in zip(got, (dg @ s["wg"] + du @ s["wu"], dg.T @ s["x"], du.T @ s["x"])):
                    assert torch.equal(torch.isnan(g), torch.isnan(r)), (act, name, bad)
                    assert torch.equal(torch.where(torch.isinf(g), g.double(), 0.0), torch.where(torch.isinf(r), r, 0.0)), (act, name, bad)
    assert rd.rd_block_status() == rd.RD_OK


@gpu
@pytest.mark.parametrize("n, dim, width", [(40, 72, 150), (300, 520, 77)])
def test_gated_grad_range_of_fp16(n, dim, width):
    """dgate and dup are operands in the matrices' type: in fp16 above 65504 infinite, also where the gradients would fit, and below 2^-14 in
    steps of 2^-24; in bf16 they have fp32's range."""
    i, j = n // 2, width // 2
    for dtype in HALF:
        x, wg, wu = rand(n, dim, seed=1, dtype=dtype), rand(width, dim, seed=2, dtype=dtype, std=0.01), rand(width, dim, seed=3, dtype=dtype, std=0.01)
        gate, up, d = (rand(n, width, seed=4 + k, dtype=dtype) for k in range(3))
        gate[i, j], up[i, j], d[i, j] = 3.0, 400.0, 200.0                       # dgate 8.3e4, dup 571
        (dx, ex), *weights = grad_reference(*(t.double() for t in (d, x, wg, wu, gate, up)), rd.RD_SILU, dtype)
        assert dx.abs().max() < 6e3 and all(w.abs().max() < 4e5 for w, _ in weights)
        gx, gg, gu = rd.rd_gated_grad(d, x, wg, wu, gate, up)
        rest = torch.arange(n, device="cuda") != i
        if dtype == torch.float16:
            assert torch.isinf(gx[i]).all() and torch.isinf(gg[j]).all() and torch.isfinite(gx[rest]).all() and torch.isfinite(gu).all()
        else:
            within(gx, dx, ex + U[dtype] * (dx.abs() + ex) + TINY[dtype])
            within(gg, weights[0][0], weights[0][1] + U[dtype] * (weights[0][0].abs() + weights[0][1]) + TINY[dtype])
        # small gradients of ordinary values, half of them below the normal numbers: off by half a step of 2^-24 each, as grad_reference has it
        small = (rand(n, width, seed=8, dtype=torch.float32) * 2.0 ** -13).to(dtype)
        up[i, j] = 1.0
        want = grad_reference(*(t.double() for t in (small, x, wg, wu, gate, up)), rd.RD_SILU, dtype)
        for g, (w, e) in zip(rd.rd_gated_grad(small, x, wg, wu, gate, up), want):
            within(g, w, e + U[dtype] * (w.abs() + e) + TINY[dtype])
