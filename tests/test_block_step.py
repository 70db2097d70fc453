"""The operators together: a training step with feed-forward blocks over processes, and the serving path from the norm's 8 bits into
the gated projections."""
import math

import pytest
import torch

import paper_1310_4645_b200 as rd
from test_gated import activation
from test_norm import BF16, E4M3, kept, norm_reference
from test_vocab import U, ints, rand, within

gpu = pytest.mark.gpu


def norm64(x, w, eps):
    return x * (x.square().mean(1, keepdim=True) + eps).rsqrt() * w


@gpu
@pytest.mark.parametrize("processes, blocks, drop, act", [(1, 1, 0.0, rd.RD_SILU), (4, 2, 0.2, rd.RD_SILU), (2, 1, 0.5, rd.RD_GELU), (3, 3, 0.1, rd.RD_RELU)])
def test_step_with_blocks(processes, blocks, drop, act):
    """A step over processes against the same step in 64 bits, derived by autograd."""
    from paper_1310_4645_b200.vocab_step import VocabStep
    rows, dim, width, n = 96 * processes, 72, 40 * processes, 70
    table = rand(rows, dim, seed=1, dtype=BF16, std=0.3)
    layers = [((1 + rand(1, dim, seed=10 * k, std=0.2)[0]), rand(width, dim, seed=10 * k + 1, dtype=BF16, std=dim ** -0.5),
               rand(width, dim, seed=10 * k + 2, dtype=BF16, std=dim ** -0.5), rand(dim, width, seed=10 * k + 3, dtype=BF16, std=width ** -0.5)) for k in range(1, blocks + 1)]
    final = 1 + rand(1, dim, seed=2, std=0.2)[0]
    ids, labels = ints(0, rows, n, seed=3), ints(0, rows, n, seed=4)
    labels[::5] = -100
    step = VocabStep(table, processes, n, blocks=layers, final_norm=final, drop=drop, activation=act)
    try:
        loss, grads = step.run(ids, labels, embed_scale=3.0, logit_scale=0.2, z_loss=1e-3, seed=77, step=5)
        mask = lambda layer: kept(n, dim, drop, 77, 5 * (blocks + 1) + layer) if drop else 1.0
        w = table.double().requires_grad_()
        leaves = [[t.double().requires_grad_() for t in layer] for layer in layers]
        last = final.double().requires_grad_()
        stream, result = w[ids] * 3.0 * mask(0), None
        for k, (norm, gate, up, down) in enumerate(leaves):
            if result is not None:
                stream = stream + result * mask(k)
            h = norm64(stream, norm, 1e-6)
            result = (activation(act, h @ gate.T)[0] * (h @ up.T)) @ down.T
        stream = stream + result * mask(blocks)
        x = norm64(stream, last, 1e-6) @ w.T * 0.2
        lse = torch.logsumexp(x, 1)
        counts = labels >= 0
        target = x.gather(1, labels.clamp(min=0)[:, None])[:, 0]
        want = torch.where(counts, lse - target + 1e-3 * lse * lse, 0.0).sum() / counts.sum()
        want.backward()
        # every value on the way is rounded to 16 bits some six times a block and five times at the ends, each 2^-8 of it at most; of
        # logits of this size the loss inherits that absolutely, gradients of either sign inherit it relative to their norm
        rounds = (6 * blocks + 5) * U[BF16]
        size = x.abs().max().item()
        assert abs(loss.item() - want.item()) <= rounds * size
        bound = rounds * (1 + size)
        near = lambda got, ref: (got.double() - ref).norm().item() <= bound * ref.norm().item()
        assert near(torch.cat(grads), w.grad) and near(step.final_norm_grad, last.grad)
        for block, (norm, gate, up, down) in zip(step.blocks, leaves):
            assert near(block.grads[0], norm.grad) and near(torch.cat(block.grads[1]), gate.grad) and near(torch.cat(block.grads[2]), up.grad)
            assert near(torch.cat(block.grads[3], 1), down.grad)
        # the same step again, the same bits; another step, other masks
        first = [g.clone() for _, g in step.parameters()]
        step.run(ids, labels, embed_scale=3.0, logit_scale=0.2, z_loss=1e-3, seed=77, step=5)
        assert all(torch.equal(a, g) for a, (_, g) in zip(first, step.parameters()))
        if drop:
            step.run(ids, labels, embed_scale=3.0, logit_scale=0.2, z_loss=1e-3, seed=77, step=6)
            assert not torch.equal(first[0], step.grads[0])
        assert rd.rd_block_status() == rd.RD_OK and rd.rd_vocab_status() == rd.RD_OK
    finally:
        step.close()


@gpu
def test_step_command_with_blocks(capsys):
    from paper_1310_4645_b200 import vocab_step
    vocab_step.main(["--processes", "2", "--vocab", "512", "--dim", "64", "--tokens", "100", "--steps", "3", "--blocks", "2", "--width", "128", "--rate", "0.1"])
    losses = [float(line.split()[3]) for line in capsys.readouterr().out.splitlines()]
    assert len(losses) == 3 and all(map(math.isfinite, losses))


@gpu
def test_step_needs_its_parts():
    from paper_1310_4645_b200.vocab_step import VocabStep
    table = torch.zeros(64, 8, device="cuda", dtype=BF16)
    layer = (torch.ones(8, device="cuda"), torch.zeros(9, 8, device="cuda", dtype=BF16), torch.zeros(9, 8, device="cuda", dtype=BF16), torch.zeros(8, 9, device="cuda", dtype=BF16))
    for kw in (dict(blocks=[layer], final_norm=layer[0]), dict(final_norm=layer[0])):
        with pytest.raises(ValueError):
            VocabStep(table, 2, 4, **kw)


@gpu
@pytest.mark.parametrize("n", [1, 3, 60, 300])
def test_norm_into_gated_in_8bit(n):
    """A serving step: residual, norm into 8 bits, gated projections of 8-bit weights, against 64 bits on the values that the 8 bits
    stand for, and against the step without them."""
    dim, width = 256, 520
    x, residual, weight = rand(n, dim, seed=20, dtype=BF16), rand(n, dim, seed=21), 1 + rand(1, dim, seed=22, std=0.2)[0]

    def eight(rows, seed):
        t = rand(rows, dim, seed=seed, std=dim ** -0.5)
        scale = t.abs().amax(1) / 448
        return (t / scale[:, None]).to(E4M3), scale

    (wg, sg), (wu, su) = eight(width, 23), eight(width, 24)
    q, total, rstd, scale = rd.rd_norm(x, weight, residual, out_dtype=E4M3)
    out, _, _ = rd.rd_gated(q, wg, wu, x_scale=scale, gate_scale=sg, up_scale=su)
    s, _, r, _ = norm_reference(x, weight, residual, 1e-6, 1.0)
    value = lambda t, k: t.float().double() * k.double()[:, None]
    h, g64, u64 = value(q, scale), value(wg, sg), value(wu, su)
    g, u = h @ g64.T, h @ u64.T
    v, _, ev, _ = activation(rd.RD_SILU, g)
    # products exact, sums of dim terms, the scales' products: the bound of the projections alone
    eg, eu = ((h.abs() @ w.abs().T) * (dim + 8) * 2.0 ** -23 for w in (g64, u64))
    bound = (ev + 1.13 * eg) * (u.abs() + eu) + v.abs() * eu + 2.0 ** -23 * (v * u).abs()
    within(out, v * u, bound + U[BF16] * ((v * u).abs() + bound) + 2.0 ** -133)
    # the rounding to 8 bits: each term of a sum off by 2^-4 of its row's values at most, on average over dim terms of either sign far less
    exact = (s * r[:, None] * weight.double())
    g0, u0 = exact @ g64.T, exact @ u64.T
    want = activation(rd.RD_SILU, g0)[0] * u0
    assert (out.double() - want).norm() <= 2 * 2.0 ** -4 * want.norm() + U[BF16] * want.norm()
