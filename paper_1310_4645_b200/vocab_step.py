"""The vocabulary's part of a training step, cut over p processes and joined by this library's reductions.

    python -m paper_1310_4645_b200.vocab_step [--processes 4] [--vocab 32768] [--dim 1024] [--tokens 2048] [--steps 5]

Process i (a buffer of this GPU, as everywhere in this library) holds an equal slice of a table that serves as embedding and as
output matrix.  A step: every process looks up the tokens of its slice (rd_embed), the partial embeddings are summed
(rd_allreduce); softmax statistics of every slice (rd_vocab_loss) are joined by a max and two sums; gradients of every slice
(rd_vocab_loss_grad), those of the hidden rows summed; the embedding's gradient is added to the slice's (rd_embed_grad with
accumulate).  There is no model between the two ends: every token's embedding is asked for the token's successor.
"""
from __future__ import annotations

import argparse
import math

import torch

from . import binding as rd


class VocabStep:
    """Slices of a table over `processes` buffers, and the schedules that join their results."""

    def __init__(self, table, processes, tokens, algo=None, model=(2e-6, 1e-10, 5e-11)):
        rows, dim = table.shape
        if rows % processes:
            raise ValueError("the vocabulary must be a multiple of the number of processes")
        if tokens * dim % 2:
            raise ValueError("an even number of values is needed per message")
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

    def close(self):
        rd.rd_destroy(self.rows_schedule)
        rd.rd_destroy(self.token_schedule)

    def _join(self, values, op):
        """All-reduces one fp32 vector per process; the first process's copy."""
        for i, v in enumerate(values):
            self.stat[i].copy_(v)
        rd.rd_allreduce(self.token_schedule, self.stat, self.joined, op)
        return self.joined[0].clone()

    def run(self, ids, labels, embed_scale=1.0, logit_scale=1.0, z_loss=0.0):
        """(mean loss, [gradient of every slice]) of the tokens `ids` with the labels `labels` (negative: does not count)."""
        rows = lambda buffer, i: buffer[i].view(self.n, self.dim)
        firsts = [i * self.rows for i in range(self.p)]
        for i, first in enumerate(firsts):
            rd.rd_embed(self.slices[i], ids, rows(self.partial, i), first_row=first, scale=embed_scale)
        rd.rd_allreduce(self.rows_schedule, self.partial, self.hidden, rd.RD_SUM)
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
        for i, first in enumerate(firsts):
            rd.rd_embed_grad(rows(self.grad_hidden, i), ids, self.grads[i], first_row=first, scale=embed_scale, accumulate=True)
        return loss, self.grads


def main(argv=None):
    a = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    a.add_argument("--processes", type=int, default=4)
    a.add_argument("--vocab", type=int, default=32768)
    a.add_argument("--dim", type=int, default=1024)
    a.add_argument("--tokens", type=int, default=2048)
    a.add_argument("--steps", type=int, default=5)
    a.add_argument("--rate", type=float, default=2.0)
    a = a.parse_args(argv)
    g = torch.Generator(device="cuda").manual_seed(0)
    table = torch.randn(a.vocab, a.dim, generator=g, device="cuda").mul_(1 / math.sqrt(a.dim)).bfloat16()
    text = torch.randint(0, a.vocab, (a.tokens + 1,), generator=g, device="cuda")
    ids, labels = text[:-1].contiguous(), text[1:].contiguous()
    labels[::7] = -100                                                   # say, a prompt's tokens
    step = VocabStep(table, a.processes, a.tokens)
    try:
        for k in range(a.steps):
            start, stop = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            start.record()
            loss, grads = step.run(ids, labels, embed_scale=math.sqrt(a.dim), logit_scale=1.0)
            stop.record()
            for s, grad in zip(step.slices, grads):
                s.add_(grad, alpha=-a.rate)
            print("step %d  loss %.4f  %.3f ms" % (k, loss.item(), start.elapsed_time(stop)))
        if rd.rd_vocab_status() != rd.RD_OK:
            raise SystemExit("a kernel gave up a wait")
    finally:
        step.close()


if __name__ == "__main__":
    main()
