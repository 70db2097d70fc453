"""The gradients of a training step with feed-forward blocks, closely enough that a mask or a term left out shows.

Bound.  Values and gradients are rounded to 16 bits some six times a block and five times at the ends, each off by at most 2^-8 of itself
and, over many values, by no more than 2^-8 / sqrt(3) in the mean square.  These errors have nothing to do with one another, so their
squares add up; a value may enter a gradient on two ways (gate and up, forward and back), hence twice: 2 sqrt(roundings) 2^-8 of the
gradient's norm, the 1 / sqrt(3) as the margin.  (relu is left out: a gate near 0 whose sign a rounding decides is off by all of itself.)

On the CPU a step with the same roundings stands in for the kernels': it keeps the bound, and with any one mistake planted it does not.
"""
import math

import numpy as np
import pytest
import torch

import paper_1310_4645_b200 as rd
from test_gated import activation
from test_norm import philox

gpu = pytest.mark.gpu
EPS, EMBED, LOGIT, Z_LOSS, SEED, STEP = 1e-6, 3.0, 0.2, 0.1, 77, 5
CASES = [(1, 1, 0.0, rd.RD_SILU), (4, 2, 0.2, rd.RD_SILU), (2, 1, 0.5, rd.RD_GELU), (3, 3, 0.1, rd.RD_GELU)]


def r16(t):
    return t.bfloat16().double()


class Case:
    def __init__(self, processes, blocks, drop, act):
        g = torch.Generator().manual_seed(1000 + processes)
        rand = lambda *shape, std=1.0: torch.randn(*shape, generator=g).mul_(std)
        self.processes, self.drop, self.act = processes, drop, act
        self.rows, self.dim, self.width, self.n = 96 * processes, 72, 40 * processes, 70
        self.table = rand(self.rows, self.dim, std=0.3).bfloat16()
        norm = lambda: 1 + rand(self.dim, std=0.2)
        self.layers = [(norm(), *(rand(*s, std=s[1] ** -0.5).bfloat16() for s in ((self.width, self.dim), (self.width, self.dim), (self.dim, self.width)))) for _ in range(blocks)]
        self.final = norm()
        self.ids, self.labels = (torch.randint(0, self.rows, (self.n,), generator=g) for _ in range(2))
        self.labels[::5] = -100
        self.counts = self.labels >= 0

    def mask(self, layer):
        """What dropout multiplies by, in 64 bits."""
        if not self.drop:
            return 1.0
        offset, low = STEP * (len(self.layers) + 1) + layer, np.uint64(0xFFFF)
        row, unit = np.meshgrid(np.arange(self.n, dtype=np.uint64), np.arange(self.dim // 8, dtype=np.uint64), indexing="ij")
        words = philox([unit, row, np.full_like(row, offset), np.zeros_like(row)], [np.full_like(row, SEED), np.zeros_like(row)])
        bits = np.stack([w >> np.uint64(s) & low for w in words for s in (0, 16)], -1).reshape(self.n, self.dim)
        border = round(float(np.float32(self.drop)) * 65536)
        return torch.from_numpy((bits >= border) * (65536 / (65536 - border)))

    def loss(self, logits):
        lse = torch.logsumexp(logits, 1)
        target = logits.gather(1, self.labels.clamp(min=0)[:, None])[:, 0]
        return torch.where(self.counts, lse - target + Z_LOSS * lse * lse, 0.0).sum() / self.counts.sum()


def norm64(x, w):
    return x * (x.square().mean(1, keepdim=True) + EPS).rsqrt() * w


def exact_step(c):
    """(loss, gradients by name) in 64 bits, derived by autograd."""
    w = c.table.double().requires_grad_()
    leaves = [[t.double().requires_grad_() for t in layer] for layer in c.layers]
    last = c.final.double().requires_grad_()
    stream, result = w[c.ids] * EMBED * c.mask(0), None
    for k, (norm, gate, up, down) in enumerate(leaves):
        if result is not None:
            stream = stream + result * c.mask(k)
        h = norm64(stream, norm)
        result = (activation(c.act, h @ gate.T)[0] * (h @ up.T)) @ down.T
    stream = stream + result * c.mask(len(leaves))
    loss = c.loss(norm64(stream, last) @ w.T * LOGIT)
    loss.backward()
    grads = {"table": w.grad, "final norm": last.grad}
    for k, leaf in enumerate(leaves):
        grads |= {"%s %d" % (name, k): t.grad for name, t in zip(("norm", "gate", "up", "down"), leaf)}
    return loss.item(), grads


def rounded_step(c, mistake=None):
    """The same step, forth and back by hand, rounded to 16 bits wherever the kernels round; `mistake`: what goes wrong in it."""
    p, table = c.processes, c.table.double()
    cut = lambda t, k=0: t.double().chunk(p, k)
    masks = [c.mask(k) for k in range(len(c.layers) + 1)]
    root = lambda s: (s.square().mean(1, keepdim=True) + EPS).rsqrt()
    stream = r16(r16(EMBED * table[c.ids]) * masks[0])
    result, kept = None, []
    for k, (norm, gate, up, down) in enumerate(c.layers):
        s = stream if result is None else stream + result * masks[k]
        h, stream, rstd = r16(s * root(s) * norm.double()), r16(s), root(s)
        slices, parts = [], []
        for wg, wu, wd in zip(cut(gate), cut(up), cut(down, 1)):
            g, u = h @ wg.T, h @ wu.T
            out = r16(activation(c.act, g)[0] * u)
            slices.append((wg, wu, wd, out, r16(g), r16(u)))
            parts.append(r16(out @ wd.T))
        result = r16(sum(parts))
        kept.append((h, stream, rstd, slices))
    s = stream + result * masks[-1]
    h, stream, rstd = r16(s * root(s) * c.final.double()), r16(s), root(s)
    logits = h @ table.T * LOGIT
    loss = c.loss(logits).item()

    lse = torch.logsumexp(logits, 1, keepdim=True)
    d = (logits - lse).exp() * (1 + (0.0 if mistake == "no z-loss" else 2 * Z_LOSS * lse))
    d[torch.arange(c.n), c.labels.clamp(min=0)] -= 1
    d = r16(d * c.counts[:, None] * LOGIT / c.counts.sum())
    grads = {"table": r16(d.T @ h)}
    grad = r16(sum(r16(di @ wi) for di, wi in zip(d.chunk(p, 1), cut(table))))

    def norm_back(grad, total, rstd, weight, more, mask):
        g, xhat = grad * weight.double(), total * rstd
        mean = 0.0 if mistake == "no mean in the norm's gradient" else (g * xhat).mean(1, keepdim=True)
        both = rstd * (g - xhat * mean)
        if more is not None and mistake != "no residual":
            both = both + more
        return r16(both * (1.0 if mistake == "no mask on the way back" else mask)), r16(both), (grad * xhat).sum(0)

    grad, grad_stream, grads["final norm"] = norm_back(grad, stream, rstd, c.final, None, 1.0 if mistake == "no mask of the last block on the way back" else masks[-1])
    for k in reversed(range(len(c.layers))):
        h, stream, rstd, slices = kept[k]
        parts, of_gate, of_up, of_down = [], [], [], []
        for wg, wu, wd, out, g, u in slices:
            value, slope, _, _ = activation(c.act, g)
            up = r16(grad @ wd)
            dg, du = r16(up * u * (1.0 if mistake == "no slope" else slope)), r16(up * value)
            parts.append(r16(dg @ wg + (0.0 if mistake == "no gradient through up" else du @ wu)))
            of_gate.append(r16(dg.T @ h)), of_up.append(r16(du.T @ h)), of_down.append(r16(grad.T @ out))
        if mistake == "a process left out" and p > 1:
            parts.pop()
        grads |= {"gate %d" % k: torch.cat(of_gate), "up %d" % k: torch.cat(of_up), "down %d" % k: torch.cat(of_down, 1)}
        grad, grad_stream, grads["norm %d" % k] = norm_back(r16(sum(parts)), stream, rstd, c.layers[k][0], grad_stream, masks[k] if k else 1.0)
    grad = r16(grad_stream * (1.0 if mistake in ("no mask on the way back", "no mask of the embedding on the way back") else masks[0]))
    if mistake != "no gradient of the embedding":
        grads["table"] = r16(grads["table"].index_add(0, c.ids, EMBED * grad))
    return loss, grads


def worst(c, got, want):
    """The gradients' (and the loss's) largest distance from 64 bits, in units of the bound."""
    bound = 2 * math.sqrt(6 * len(c.layers) + 5) * 2.0 ** -8
    assert got[1].keys() == want[1].keys()
    off = {name: ((got[1][name].double().cpu() - g).norm() / g.norm()).item() / bound for name, g in want[1].items()}
    off["loss"] = abs(got[0] - want[0]) / abs(want[0]) / bound
    return max(off.values())


@pytest.mark.parametrize("processes, blocks, drop, act", CASES)
def test_the_bound_shows_mistakes(processes, blocks, drop, act):
    c = Case(processes, blocks, drop, act)
    want = exact_step(c)
    assert worst(c, rounded_step(c), want) <= 1
    mistakes = ["no z-loss", "no mean in the norm's gradient", "no residual", "no slope", "no gradient through up", "no gradient of the embedding"]
    mistakes += ["no mask on the way back", "no mask of the last block on the way back", "no mask of the embedding on the way back"] if drop else []
    mistakes += ["a process left out"] if processes > 1 else []
    for mistake in mistakes:
        assert worst(c, rounded_step(c, mistake), want) > 1, mistake


@gpu
@pytest.mark.parametrize("processes, blocks, drop, act", CASES)
def test_step_with_blocks_closely(processes, blocks, drop, act):
    from paper_1310_4645_b200.vocab_step import VocabStep
    c = Case(processes, blocks, drop, act)
    step = VocabStep(c.table.cuda(), processes, c.n, blocks=[[t.cuda() for t in layer] for layer in c.layers], final_norm=c.final.cuda(), drop=drop, activation=act, eps=EPS)
    try:
        loss, grads = step.run(c.ids.cuda(), c.labels.cuda(), embed_scale=EMBED, logit_scale=LOGIT, z_loss=Z_LOSS, seed=SEED, step=STEP)
        got = {"table": torch.cat(grads), "final norm": step.final_norm_grad}
        for k, block in enumerate(step.blocks):
            norm, gate, up, down = block.grads
            got |= {"norm %d" % k: norm, "gate %d" % k: torch.cat(gate), "up %d" % k: torch.cat(up), "down %d" % k: torch.cat(down, 1)}
        assert worst(c, (loss.item(), got), exact_step(c)) <= 1
        assert rd.rd_block_status() == rd.RD_OK and rd.rd_vocab_status() == rd.RD_OK
    finally:
        step.close()
