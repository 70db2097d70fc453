"""Cases of the vocabulary operators: embedding lookup and its gradient, softmax cross entropy over a large vocabulary and
its gradient.

A model meets its vocabulary twice: a table of `rows` x `dim` turns token ids into vectors, and the same or another such
matrix turns the last hidden vectors into logits for the loss.  `first` is the first vocabulary entry of the rows that a
process holds when the vocabulary is cut into `shards` equal pieces, one per process (0 and 1 when it is not).
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
SIZE = {"bf16": 2, "fp16": 2, "fp32": 4}


def listed():
    return [
        # one token of a decoding step looked up: nothing but latency
        {"name": "embed-1", "op": "embed", "n": 1, "rows": 32768, "dim": 1024, "dtype": "bf16", "scale": 32.0, "shards": 1},
        # a training batch, rows scaled by sqrt(dim)
        {"name": "embed-16384", "op": "embed", "n": 16384, "rows": 131072, "dim": 4096, "dtype": "bf16", "scale": 64.0, "shards": 1},
        # a short fine-tuning batch with odd sizes, gradient kept in 32 bits
        {"name": "embed-grad-257", "op": "embed_grad", "n": 257, "rows": 10007, "dim": 520, "dtype": "fp16", "out": "fp32", "scale": 1.0, "shards": 1},
        # a training batch: the dense gradient of the whole table
        {"name": "embed-grad-16384", "op": "embed_grad", "n": 16384, "rows": 131072, "dim": 4096, "dtype": "bf16", "out": "bf16", "scale": 64.0, "shards": 1},
        # a long batch on a process that holds a quarter of the vocabulary, gradient in 32 bits
        {"name": "embed-grad-shard", "op": "embed_grad", "n": 65536, "rows": 32768, "dim": 2048, "dtype": "bf16", "out": "fp32", "scale": 1.0, "shards": 4},
        # the log-probability of one token
        {"name": "loss-1", "op": "loss", "n": 1, "rows": 32768, "dim": 1024, "dtype": "bf16", "scale": 1.0, "z": 0.0, "ignored": 0.0, "shards": 1},
        # a fine-tuning batch whose prompt tokens are ignored, odd sizes, with the penalty on the normaliser
        {"name": "loss-2000", "op": "loss", "n": 2000, "rows": 50021, "dim": 1000, "dtype": "fp16", "scale": 1.0, "z": 1e-4, "ignored": 0.3, "shards": 1},
        # a training batch
        {"name": "loss-8192", "op": "loss", "n": 8192, "rows": 131072, "dim": 4096, "dtype": "bf16", "scale": 1.0, "z": 0.0, "ignored": 0.0, "shards": 1},
        # a byte-level vocabulary's size of model, few tokens: latency
        {"name": "loss-grad-37", "op": "loss_grad", "n": 37, "rows": 1009, "dim": 256, "dtype": "bf16", "scale": 1.0, "z": 0.0, "ignored": 0.0, "shards": 1},
        # few tokens on a large vocabulary: the matrices' bytes count, not the products
        {"name": "loss-grad-128", "op": "loss_grad", "n": 128, "rows": 131072, "dim": 4096, "dtype": "bf16", "scale": 0.5, "z": 1e-4, "ignored": 0.0, "shards": 1},
        # a fine-tuning batch on half the vocabulary, ignored tokens, an odd number of rows
        {"name": "loss-grad-4096", "op": "loss_grad", "n": 4096, "rows": 32003, "dim": 2048, "dtype": "fp16", "scale": 1.0, "z": 0.0, "ignored": 0.4, "shards": 2},
        # a training batch
        {"name": "loss-grad-8192", "op": "loss_grad", "n": 8192, "rows": 131072, "dim": 4096, "dtype": "bf16", "scale": 1.0, "z": 0.0, "ignored": 0.0, "shards": 1},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["embed", "embed_grad", "loss", "loss_grad"])
    while True:
        dim = _log(rng, 64, 4096)
        if rng.random() < 0.75:
            dim = max(64, dim // 64 * 64)
        rows = _log(rng, 1000, 131072)
        n = _log(rng, 1, 65536 if op.startswith("embed") else 8192)
        if 3072 not in (dim, rows, n) and n * dim <= 16384 * 4096:
            break
    case = {"op": op, "n": n, "rows": rows, "dim": dim, "shards": rng.choice([1, 1, 1, 2, 4])}
    if op.startswith("embed"):
        case["dtype"] = rng.choice(["bf16", "bf16", "fp16", "fp32"])
        case["scale"] = rng.choice([1.0, math.sqrt(dim)])
        if op == "embed_grad":
            case["out"] = rng.choice([case["dtype"], "fp32"])
    else:
        case["dtype"] = rng.choice(["bf16", "bf16", "fp16"])
        case["scale"] = rng.choice([1.0, 0.5])
        case["z"] = rng.choice([0.0, 1e-4])
        case["ignored"] = rng.choice([0.0, 0.0, 0.3, 0.5])
    return case


def _first(case):
    return case["rows"] if case["shards"] > 1 else 0        # the second shard, where there are several


def _tokens(case, g):
    """Token ids of the whole vocabulary, about as frequent as words are (the k-th most frequent in proportion to 1/k)."""
    total = case["rows"] * case["shards"]
    k = torch.exp(torch.rand(case["n"], generator=g, device="cuda", dtype=torch.float64) * math.log(total + 1)).long() - 1
    return (k.clamp_(0, total - 1) * 7919 + 13) % total


def _distinct(case):
    """How many different rows of the process's shard a batch is expected to touch."""
    total = case["rows"] * case["shards"]
    k = np.arange(total, dtype=np.float64)
    p = np.log((k + 2) / (k + 1)) / math.log(total + 1)
    return float((1 - (1 - p) ** case["n"]).sum()) / case["shards"]


def _valid(case):
    return case["n"] - int(case["n"] * case.get("ignored", 0.0))


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    n, rows, dim, dtype = case["n"], case["rows"], case["dim"], DTYPES[case["dtype"]]
    ids = _tokens(case, g)
    state = {"case": case, "ids": ids, "first": _first(case)}
    if case["op"] == "embed":
        state["table"] = torch.randn(rows, dim, generator=g, device="cuda").mul_(0.02).to(dtype)
    elif case["op"] == "embed_grad":
        state["grad"] = torch.randn(n, dim, generator=g, device="cuda").mul_(1e-2).to(dtype)
    else:
        weight = torch.randn(rows, dim, generator=g, device="cuda").mul_(2.5 / math.sqrt(dim)).to(dtype)
        hidden = torch.randn(n, dim, generator=g, device="cuda")
        # a model that has learnt something: half of the tokens lean towards their label's row
        local = (ids - state["first"]).clamp(0, rows - 1)
        lean = (torch.rand(n, 1, generator=g, device="cuda") < 0.5) * 1.2
        hidden = (hidden + lean * weight[local].float()).to(dtype)
        out = torch.randperm(n, generator=g, device="cuda")[: n - _valid(case)]
        ids[out] = -100
        state |= {"weight": weight, "hidden": hidden}
        if case["op"] == "loss_grad":
            w = weight.float()
            lse = torch.cat([torch.logsumexp(h.float() @ w.T * case["scale"], 1) for h in hidden.split(2048)])
            # the other shards' part of the normaliser
            state["lse"] = lse + math.log(case["shards"])
            # the mean over the tokens that count, some of them weighted
            weights = 0.5 + torch.rand(n, generator=g, device="cuda")
            state["grad_loss"] = weights / max(1, _valid(case))
    return state


def _plain_embed(table, ids, first, scale):
    at = ids - first
    inside = (at >= 0) & (at < table.shape[0])
    return (table[torch.where(inside, at, 0)].float() * (inside[:, None] * scale)).to(table.dtype)


def _plain_embed_grad(grad, ids, rows, first, scale, dtype):
    at = ids - first
    inside = (at >= 0) & (at < rows)
    out = torch.zeros(rows + 1, grad.shape[1], device=grad.device)
    out.index_add_(0, torch.where(inside, at, rows), grad.float() * scale)
    return out[:rows].to(dtype)


def _plain_loss(hidden, weight, ids, first, scale, z):
    x = (hidden.float() @ weight.float().T) * scale
    most = x.amax(1)
    lse = most + (x - most[:, None]).exp().sum(1).log()
    at = ids - first
    here = (at >= 0) & (at < weight.shape[0]) & (ids >= 0)
    target = torch.where(here, x.gather(1, torch.where(here, at, 0)[:, None])[:, 0], 0.0)
    counts = ids >= 0
    lse = torch.where(counts, lse, 0.0)
    return torch.where(counts, lse - target + z * lse * lse, 0.0), lse, target


def _plain_loss_grad(hidden, weight, ids, first, scale, z, lse, grad_loss):
    h, w = hidden.float(), weight.float()
    d = ((h @ w.T) * scale - lse[:, None]).exp()
    at = ids - first
    here = (at >= 0) & (at < weight.shape[0]) & (ids >= 0)
    g = torch.where(ids >= 0, grad_loss, 0.0)
    d *= (g * (1 + 2 * z * lse))[:, None]
    rows = torch.arange(len(ids), device=ids.device)
    d[rows, torch.where(here, at, 0)] -= torch.where(here, g, 0.0)
    d *= scale
    return (d @ w).to(hidden.dtype), (d.T @ h).to(weight.dtype)


def run(state):
    case, first = state["case"], state["first"]
    if own:
        import paper_1310_4645_b200 as rd
        if case["op"] == "embed":
            return rd.rd_embed(state["table"], state["ids"], first_row=first, scale=case["scale"])
        if case["op"] == "embed_grad":
            out = torch.empty(case["rows"], case["dim"], dtype=DTYPES[case["out"]], device="cuda")
            return rd.rd_embed_grad(state["grad"], state["ids"], out, first_row=first, scale=case["scale"])
        if case["op"] == "loss":
            return rd.rd_vocab_loss(state["hidden"], state["weight"], state["ids"], first_row=first, scale=case["scale"], z_loss=case["z"])
        grad_hidden, grad_weight = torch.empty_like(state["hidden"]), torch.empty_like(state["weight"])
        return rd.rd_vocab_loss_grad(state["hidden"], state["weight"], state["ids"], state["lse"], state["grad_loss"], grad_hidden, grad_weight,
                                     first_row=first, scale=case["scale"], z_loss=case["z"])
    if case["op"] == "embed":
        return _plain_embed(state["table"], state["ids"], first, case["scale"])
    if case["op"] == "embed_grad":
        return _plain_embed_grad(state["grad"], state["ids"], case["rows"], first, case["scale"], DTYPES[case["out"]])
    if case["op"] == "loss":
        return _plain_loss(state["hidden"], state["weight"], state["ids"], first, case["scale"], case["z"])
    return _plain_loss_grad(state["hidden"], state["weight"], state["ids"], first, case["scale"], case["z"], state["lse"], state["grad_loss"])


def work(case):
    n, rows, dim, size = case["n"], case["rows"], case["dim"], SIZE[case["dtype"]]
    if case["op"] == "embed":
        return {"bytes": 8 * n + (_distinct(case) + n) * dim * size, "flops": n * dim}
    if case["op"] == "embed_grad":
        here = n / case["shards"]
        return {"bytes": 8 * n + here * dim * size + rows * dim * SIZE[case["out"]], "flops": here * dim}
    m = _valid(case)
    if case["op"] == "loss":
        return {"bytes": 8 * n + (m + rows) * dim * size + 12 * n, "flops": 2 * m * rows * dim}
    return {"bytes": 16 * n + (m + rows) * dim * size + (n + rows) * dim * size, "flops": 6 * m * rows * dim}


def exact(case, seed):
    """The definition, token by token and row by row, in 64 bits."""
    s = prepare(case, seed)
    n, rows, scale = case["n"], case["rows"], float(case["scale"])
    label = s["ids"] - s["first"]
    mine = (s["ids"] >= 0) & (label >= 0) & (label < rows)
    if case["op"] == "embed":
        out = torch.zeros(n, case["dim"], dtype=torch.float64, device="cuda")
        out[mine] = s["table"].double()[label[mine]] * scale
        return out
    if case["op"] == "embed_grad":
        # sorted by row, differences of a running sum at the rows' ends
        kept = torch.nonzero(mine)[:, 0]
        order = kept[torch.sort(label[kept], stable=True).indices]
        count = torch.bincount(label[kept], minlength=rows)
        out = torch.empty(rows, case["dim"], dtype=torch.float64, device="cuda")
        for c in range(0, case["dim"], 512):
            run_sum = torch.cumsum(s["grad"][order, c:c + 512].double(), 0)
            run_sum = torch.cat([run_sum.new_zeros(1, run_sum.shape[1]), run_sum])
            ends = torch.cumsum(count, 0)
            out[:, c:c + 512] = (run_sum[ends] - run_sum[ends - count]) * scale
        return out
    weight = s["weight"].double()
    loss, lses, targets, grads = [], [], [], []
    grad_weight = torch.zeros_like(weight) if case["op"] == "loss_grad" else None
    for b in range(0, n, 1024):
        e = min(n, b + 1024)
        h = s["hidden"][b:e].double()
        logits = torch.mm(h, weight.t()).mul_(scale)
        counts = (s["ids"][b:e] >= 0).double()
        hot = torch.nonzero(mine[b:e])[:, 0]
        if case["op"] == "loss":
            lse = torch.logsumexp(logits, dim=1) * counts
            target = torch.zeros(e - b, dtype=torch.float64, device="cuda")
            target[hot] = logits[hot, label[b:e][hot]]
            loss.append((lse + case["z"] * lse.square() - target) * counts)
            lses.append(lse)
            targets.append(target)
        else:
            lse, up = s["lse"][b:e].double(), s["grad_loss"][b:e].double() * counts
            p = logits.sub_(lse[:, None]).exp_()
            p *= (up + 2 * case["z"] * up * lse)[:, None]
            p[hot, label[b:e][hot]] -= up[hot]
            p *= scale
            grads.append(torch.mm(p, weight))
            grad_weight += torch.mm(p.t(), h)
    if case["op"] == "loss":
        return torch.cat(loss), torch.cat(lses), torch.cat(targets)
    return torch.cat(grads), grad_weight
