"""A training step on a vocabulary, with or without feed-forward blocks between its ends, cut over p processes and joined by this
library's reductions.

    python -m paper_1310_4645_b200.vocab_step [--processes 4] [--vocab 32768] [--dim 1024] [--tokens 2048] [--steps 5]
                                              [--blocks 0] [--width 4096] [--drop 0.1]

Process i (a buffer of this GPU, as everywhere in this library) holds an equal slice of a table that serves as embedding and as
output matrix.  A step: every process looks up the tokens of its slice (rd_embed), the partial embeddings are summed
(rd_allreduce); softmax statistics of every slice (rd_vocab_loss) are joined by a max and two sums; gradients of every slice
(rd_vocab_loss_grad), those of the hidden rows summed; the embedding's gradient is added to the slice's (rd_embed_grad with
accumulate).  Every token's embedding is asked for the token's successor.

With blocks the embedding goes through dropout (rd_dropout) into a residual stream, and every block through a norm (rd_norm) and gated
projections, of which process i holds an equal slice of the width (rd_gated), and the matching columns of the projection back
(a plain product); the processes' partial sums are joined (rd_allreduce), and the next norm adds them, after dropout, to the stream.
The gradients go the same way back (rd_norm_grad, rd_gated_grad).  What every process would compute alike, norms and dropout of
joined rows, is computed once here.
"""
from __future__ import annotations

import argparse
import math

import torch

from . import binding as rd


class Block:
    """A feed-forward block: norm [dim], gate and up [width, dim], down [dim, width], the last three in slices over the processes;
    after a step grads holds their gradients (norm, then a list of slices for each of the others)."""

    def __init__(self, norm, gate, up, down, processes):
        if gate.shape[0] % processes:
            raise ValueError("the width must be a multiple of the number of processes")
        self.norm, self.grads = norm, None
        self.gate, self.up = ([s.clone() for s in w.chunk(processes)] for w in (gate, up))
        self.down = [s.contiguous() for s in down.chunk(processes, 1)]


class VocabStep:
    """Slices of a table over `processes` buffers, and the schedules that join their results.  blocks: (norm, gate, up, down) of every
    feed-forward block; final_norm: the last norm's weight, before the loss (where there are blocks); drop: share of values that
    dropout takes from the embedding and from every block's result, activation: RD_SILU, RD_GELU or RD_RELU."""

    def __init__(self, table, processes, tokens, algo=None, model=(2e-6, 1e-10, 5e-11), blocks=(), final_norm=None, drop=0.0, activation=rd.RD_SILU, eps=1e-6):
        rows, dim = table.shape
        if rows % processes:
            raise ValueError("the vocabulary must be a multiple of the number of processes")
        if tokens * dim % 2:
            raise ValueError("an even number of values is needed per message")
        self.blocks = [Block(*b, processes) for b in blocks]
        if (final_norm is None) != (not self.blocks):
            raise ValueError("final_norm goes with blocks")
        self.slices = [s.clone() for s in table.chunk(processes)]
        self.p, self.n, self.dim, self.rows = processes, tokens, dim, rows // processes
        algo = rd.RD_UNI_GREEDY if algo is None else algo
        port = rd.RD_PORT_BI if algo in (rd.RD_BI_GREEDY, rd.RD_BUTTERFLY) else rd.RD_PORT_UNI
        self.rows_schedule = rd.rd_schedule_create(algo, port, processes, tokens * dim * table.element_size(), 0, *model)
        self.token_schedule = rd.rd_schedule_create(algo, port, processes, tokens * 4, 0, *model)
        # one buffer per process and message, and one copy of the result
        self.partial, self.hidden = (torch.empty(processes, tokens * dim, dtype=table.dtype, device=table.device) for _ in range(2))
        self.grad_part, self.grad_hidden = torch.empty_like(self.partial), torch.empty_like(self.partial)
        self.stat, self.joined = (torch.empty(processes, tokens, device=table.device) for _ in range(2))
        self.grads = [torch.empty_like(s) for s in self.slices]
        self.final_norm, self.final_norm_grad = final_norm, None
        self.drop, self.activation, self.eps = drop, activation, eps

    def close(self):
        rd.rd_destroy(self.rows_schedule)
        rd.rd_destroy(self.token_schedule)

    def _join(self, values, op):
        """All-reduces one fp32 vector per process; the first process's copy."""
        for i, v in enumerate(values):
            self.stat[i].copy_(v)
        rd.rd_allreduce(self.token_schedule, self.stat, self.joined, op)
        return self.joined[0].clone()

    def _rows(self, buffer, i):
        return buffer[i].view(self.n, self.dim)

    def _forward(self, seed, step):
        """The blocks, from the joined embeddings on; what the way back needs.  The last norm's output takes the embeddings' place."""
        layers = len(self.blocks) + 1
        drop = lambda layer: dict(drop=self.drop, seed=seed, offset=step * layers + layer)
        stream = rd.rd_dropout(self._rows(self.hidden, 0), **drop(0))
        result, kept = None, []
        for layer, block in enumerate(self.blocks):
            if result is None:
                h, _, rstd, _ = rd.rd_norm(stream, block.norm, eps=self.eps)
            else:
                h, stream, rstd, _ = rd.rd_norm(result, block.norm, stream, eps=self.eps, **drop(layer))
            projected = []
            for i in range(self.p):
                out, gate, up = rd.rd_gated(h, block.gate[i], block.up[i], self.activation, keep=True)
                torch.matmul(out, block.down[i].T, out=self._rows(self.partial, i))
                projected.append((out, gate, up))
            rd.rd_allreduce(self.rows_schedule, self.partial, self.hidden, rd.RD_SUM)
            result = self._rows(self.hidden, 0).clone()
            kept.append((h, stream, rstd, projected))
        h, stream, rstd, _ = rd.rd_norm(result, self.final_norm, stream, eps=self.eps, **drop(layers - 1))
        for i in range(self.p):
            self._rows(self.hidden, i).copy_(h)
        return kept, stream, rstd, drop

    def _backward(self, kept, stream, rstd, drop):
        """The blocks' gradients, from those of the last norm's output (joined) on; the embeddings' gradients take their place."""
        layers = len(self.blocks) + 1
        grad, grad_stream, self.final_norm_grad = rd.rd_norm_grad(self._rows(self.grad_hidden, 0), stream, self.final_norm, rstd, **drop(layers - 1))
        for layer in reversed(range(len(self.blocks))):
            block, (h, stream, rstd, projected) = self.blocks[layer], kept[layer]
            slices = []
            for i, (out, gate, up) in enumerate(projected):
                grad_down = grad.T @ out
                _, grad_gate, grad_up = rd.rd_gated_grad(grad @ block.down[i], h, block.gate[i], block.up[i], gate, up, self.activation,
                                                         grad_x=self._rows(self.grad_part, i))
                slices.append((grad_gate, grad_up, grad_down))
            rd.rd_allreduce(self.rows_schedule, self.grad_part, self.grad_hidden, rd.RD_SUM)
            more = drop(layer) if layer else {}                          # the first norm is of the stream alone
            grad, grad_stream, grad_norm = rd.rd_norm_grad(self._rows(self.grad_hidden, 0), stream, block.norm, rstd, grad_stream, **more)
            block.grads = (grad_norm, *map(list, zip(*slices)))
        grad = rd.rd_dropout(grad_stream, **drop(0))
        for i in range(self.p):
            self._rows(self.grad_hidden, i).copy_(grad)

    def run(self, ids, labels, embed_scale=1.0, logit_scale=1.0, z_loss=0.0, seed=0, step=0):
        """(mean loss, [gradient of every slice]) of the tokens `ids` with the labels `labels` (negative: does not count).  seed, step: of
        dropout; the blocks' gradients are in blocks[k].grads and final_norm_grad."""
        rows = self._rows
        firsts = [i * self.rows for i in range(self.p)]
        for i, first in enumerate(firsts):
            rd.rd_embed(self.slices[i], ids, rows(self.partial, i), first_row=first, scale=embed_scale)
        rd.rd_allreduce(self.rows_schedule, self.partial, self.hidden, rd.RD_SUM)
        kept = self._forward(seed, step) if self.blocks else None
        args = dict(scale=logit_scale, z_loss=z_loss)
        stats = [rd.rd_vocab_loss(rows(self.hidden, i), self.slices[i], labels, first_row=first, **args) for i, first in enumerate(firsts)]
        top = self._join([s[1] for s in stats], rd.RD_MAX)
        lse = top + self._join([(s[1] - top).exp() for s in stats], rd.RD_SUM).log()
        target = self._join([s[2] for s in stats], rd.RD_SUM)
        counts = labels >= 0
        weight = 1.0 / counts.sum().clamp(min=1)                        # one upstream gradient for all tokens: the mean's
        loss = (torch.where(counts, lse - target + z_loss * lse * lse, 0.0)).sum() * weight
        for i, first in enumerate(firsts):
            rd.rd_vocab_loss_grad(rows(self.hidden, i), self.slices[i], labels, lse, weight, rows(self.grad_part, i), self.grads[i], first_row=first, **args)
        rd.rd_allreduce(self.rows_schedule, self.grad_part, self.grad_hidden, rd.RD_SUM)
        if kept:
            self._backward(*kept)
        for i, first in enumerate(firsts):
            rd.rd_embed_grad(rows(self.grad_hidden, i), ids, self.grads[i], first_row=first, scale=embed_scale, accumulate=True)
        return loss, self.grads

    def parameters(self):
        """(parameter, gradient) of everything, after a step."""
        yield from zip(self.slices, self.grads)
        for b in self.blocks:
            yield b.norm, b.grads[0]
            for w, g in zip((b.gate, b.up, b.down), b.grads[1:]):
                yield from zip(w, g)
        if self.blocks:
            yield self.final_norm, self.final_norm_grad


def main(argv=None):
    a = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    a.add_argument("--processes", type=int, default=4)
    a.add_argument("--vocab", type=int, default=32768)
    a.add_argument("--dim", type=int, default=1024)
    a.add_argument("--tokens", type=int, default=2048)
    a.add_argument("--steps", type=int, default=5)
    a.add_argument("--rate", type=float, default=2.0)
    a.add_argument("--blocks", type=int, default=0)
    a.add_argument("--width", type=int, default=4096)
    a.add_argument("--drop", type=float, default=0.1)
    a = a.parse_args(argv)
    g = torch.Generator(device="cuda").manual_seed(0)
    table = torch.randn(a.vocab, a.dim, generator=g, device="cuda").mul_(1 / math.sqrt(a.dim)).bfloat16()
    text = torch.randint(0, a.vocab, (a.tokens + 1,), generator=g, device="cuda")
    ids, labels = text[:-1].contiguous(), text[1:].contiguous()
    labels[::7] = -100                                                   # say, a prompt's tokens
    matrix = lambda rows, cols: torch.randn(rows, cols, generator=g, device="cuda").mul_(1 / math.sqrt(cols)).bfloat16()
    blocks = [(torch.ones(a.dim, device="cuda"), matrix(a.width, a.dim), matrix(a.width, a.dim), matrix(a.dim, a.width)) for _ in range(a.blocks)]
    step = VocabStep(table, a.processes, a.tokens, blocks=blocks, final_norm=torch.ones(a.dim, device="cuda") if blocks else None, drop=a.drop)
    try:
        for k in range(a.steps):
            start, stop = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            start.record()
            loss, _ = step.run(ids, labels, embed_scale=math.sqrt(a.dim), logit_scale=1.0, step=k)
            stop.record()
            for weight, grad in step.parameters():
                weight.add_(grad, alpha=-a.rate)
            print("step %d  loss %.4f  %.3f ms" % (k, loss.item(), start.elapsed_time(stop)))
        if rd.rd_vocab_status() != rd.RD_OK or rd.rd_block_status() != rd.RD_OK:
            raise SystemExit("a kernel gave up a wait")
    finally:
        step.close()


if __name__ == "__main__":
    main()
