"""Values at which the block operators are easily wrong: scales whose product leaves fp32's range."""
import pytest
import torch

import paper_1310_4645_b200 as rd
from test_gated import E4M3, HALF, project
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
