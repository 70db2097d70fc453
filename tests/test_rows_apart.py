"""Rows whose beginnings are words apart and whose ends are not: a width that is not a multiple of 8 in a buffer whose stride is one, as of the
first columns of a wider matrix.  What lies between the rows belongs to somebody else: it is neither read (NaN here) nor written."""
import pytest
import torch

import paper_1310_4645_b200 as rd
from test_gated import ACTS, E4M3, HALF, outside_untouched
from test_norm import BF16, FP32
from test_vocab import gen, ints, rand

gpu = pytest.mark.gpu
WIDTHS = [1, 2, 3, 4, 5, 6, 7, 22, 63, 66, 70, 190, 253, 258, 318, 1001, 1446]


def apart(t, to=8, more=0):
    """The same values in rows that begin `to` elements' multiples apart, NaN (in 8 bits, too) between them."""
    rows, dim = t.shape
    stride = -(-dim // to) * to + more
    if t.dtype == E4M3:
        big = torch.full((rows * stride,), 0x7F, dtype=torch.uint8, device=t.device)
        view = big.view(rows, stride)[:, :dim]
        view.copy_(t.view(torch.uint8))
        return view.view(E4M3)
    view = torch.full((rows * stride,), float("nan"), dtype=t.dtype, device=t.device).view(rows, stride)[:, :dim]
    view.copy_(t)
    return view


def room(rows, dim, dtype, more=0):
    return apart(torch.full((rows, dim), 7.0, dtype=dtype, device="cuda"), more=more)


def kept_apart(results, want):
    assert all(map(torch.equal, results, want)) and all(map(outside_untouched, results))


@gpu
@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("n", [5, 200, 1300])
@pytest.mark.parametrize("dim", WIDTHS)
def test_gated_of_rows_apart(dtype, n, dim):
    for width, more in ((dim + 8, 0), (41, 8)):
        x, wg, wu = rand(n, dim, seed=1, dtype=dtype), rand(width, dim, seed=2, dtype=dtype, std=dim ** -0.5), rand(width, dim, seed=3, dtype=dtype, std=dim ** -0.5)
        d = rand(n, width, seed=4, dtype=dtype)
        act = ACTS[dim % 3]
        want = rd.rd_gated(x, wg, wu, act, keep=True)
        out = [room(n, width, dtype, more) for _ in range(3)]
        ins = [apart(t, more=more) for t in (x, wg, wu)]
        rd.rd_gated(*ins, act, out=out[0], gate=out[1], up=out[2])
        kept_apart(out, want)
        grads = rd.rd_gated_grad(d, x, wg, wu, *want[1:], act)
        into = [room(r, dim, dtype, more) for r in (n, width, width)]
        rd.rd_gated_grad(apart(d, more=more), *ins, out[1], out[2], act, grad_x=into[0], grad_gate_weight=into[1], grad_up_weight=into[2])
        kept_apart(into, grads)
    assert rd.rd_block_status() == rd.RD_OK


@gpu
@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("dim", [6, 70, 1446])
def test_gradients_side_by_side(dtype, dim):
    """Both weights' gradients as columns of one buffer, with somebody else's between them."""
    n, width = 300, 40
    x, wg, wu = rand(n, dim, seed=5, dtype=dtype), rand(width, dim, seed=6, dtype=dtype), rand(width, dim, seed=7, dtype=dtype)
    gate, up, d = (rand(n, width, seed=8 + k, dtype=dtype) for k in range(3))
    want = rd.rd_gated_grad(d, x, wg, wu, gate, up)
    buffer = rand(width, 2 * dim + 4, seed=11, dtype=dtype)                 # a multiple of 8 columns
    before = buffer.clone()
    rd.rd_gated_grad(d, x, wg, wu, gate, up, grad_gate_weight=buffer[:, :dim], grad_up_weight=buffer[:, dim + 2:2 * dim + 2])
    assert torch.equal(buffer[:, :dim], want[1]) and torch.equal(buffer[:, dim + 2:2 * dim + 2], want[2])
    assert torch.equal(buffer[:, dim:dim + 2], before[:, dim:dim + 2]) and torch.equal(buffer[:, -2:], before[:, -2:])


@gpu
@pytest.mark.parametrize("n", [5, 200])
@pytest.mark.parametrize("dim", WIDTHS)
def test_gated_8bit_of_rows_apart(n, dim):
    width = 41
    x, wg, wu = (rand(r, dim, seed=k).clamp(-3, 3).mul(100).to(E4M3) for k, r in ((1, n), (2, width), (3, width)))
    scales = dict(x_scale=torch.rand(n, generator=gen(4), device="cuda") / dim, gate_scale=torch.rand(width, generator=gen(5), device="cuda") / 100,
                  up_scale=torch.rand(width, generator=gen(6), device="cuda"))
    want = rd.rd_gated(x, wg, wu, keep=True, **scales)
    for to, more in ((16, 0), (16, 16), (8, 0)):
        out = [room(n, width, BF16, more) for _ in range(3)]
        rd.rd_gated(*(apart(t, to, more) for t in (x, wg, wu)), out=out[0], gate=out[1], up=out[2], **scales)
        kept_apart(out, want)


@gpu
@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("n, rows", [(1, 61), (3, 700), (40, 300), (200, 1000), (1500, 5000)])
@pytest.mark.parametrize("dim", WIDTHS)
def test_vocabulary_of_rows_apart(dtype, n, rows, dim):
    hidden, weight, ids = rand(n, dim, seed=1, dtype=dtype), rand(rows, dim, seed=2, dtype=dtype), ints(-1, rows, n, seed=3)
    up = torch.rand(n, generator=gen(4), device="cuda")
    for more in (0, 8):
        h, w = apart(hidden, more=more), apart(weight, more=more)
        want = rd.rd_vocab_loss(hidden, weight, ids)
        got = rd.rd_vocab_loss(h, w, ids)
        assert all(torch.allclose(a, b, rtol=1e-4, atol=1e-4) for a, b in zip(got, want))          # not the same bits: few tokens go other ways
        grads = rd.rd_vocab_loss_grad(hidden, weight, ids, want[1], up, torch.empty_like(hidden), torch.empty_like(weight))
        into = room(n, dim, dtype, more), room(rows, dim, dtype, more)
        rd.rd_vocab_loss_grad(h, w, ids, want[1], up, *into)
        for a, b in zip(into, grads):
            assert outside_untouched(a) and (a.double() - b.double()).norm() <= 0.01 * b.double().norm()
        table, looked = room(rows, dim, dtype, more), room(n, dim, dtype, more)
        rd.rd_embed(w, ids, looked)
        rd.rd_embed_grad(h, ids, table)
        kept_apart((looked, table), (rd.rd_embed(weight, ids), rd.rd_embed_grad(hidden, ids, torch.empty_like(weight))))
    assert rd.rd_vocab_status() == rd.RD_OK


@gpu
@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("dim", WIDTHS + [4099, 9001])
def test_norm_of_rows_apart(dtype, dim):
    n = 33
    x, residual, up, weight = rand(n, dim, seed=1, dtype=dtype), rand(n, dim, seed=2, dtype=dtype), rand(n, dim, seed=3, dtype=dtype), rand(1, dim, seed=4)[0]
    args = dict(drop=0.2, seed=5)
    want = rd.rd_norm(x, weight, residual, **args)
    for more in (0, 8):
        out = room(n, dim, dtype, more), room(n, dim, dtype, more)
        got = rd.rd_norm(apart(x, more=more), weight, apart(residual, more=more), out=out[0], total=out[1], **args)
        kept_apart(out, want[:2])
        grads = rd.rd_norm_grad(up, want[1], weight, want[2], residual, **args)
        into = room(n, dim, dtype, more), room(n, dim, dtype, more)
        _, _, gw = rd.rd_norm_grad(apart(up, more=more), out[1], weight, got[2], apart(residual, more=more), grad_x=into[0], grad_residual=into[1], **args)
        kept_apart(into, grads[:2])
        assert torch.equal(gw, grads[2])
        dropped = room(n, dim, dtype, more)
        rd.rd_dropout(apart(x, more=more), 0.3, 6, out=dropped)
        kept_apart([dropped], [rd.rd_dropout(x, 0.3, 6)])
