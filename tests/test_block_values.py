"""Values at which the block operators are easily wrong: scales whose product leaves fp32's range, NaN and infinities before 8 bits."""
import pytest
import torch

import paper_1310_4645_b200 as rd
from test_gated import E4M3, HALF, project
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
