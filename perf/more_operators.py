"""Cases of the feed-forward block's operators: root-mean-square norm with the residual's addition and dropout (in 16, 32 or 8
bits) and its gradient, dropout from a counter-based generator, the gated pair of projections and its gradient.

A block takes rows of `dim` values; its input projections have `width` rows each.  The residual is kept in the rows' type or in 32
bits ("sum").  `first` is the first row's number: a process that holds a slice of a batch draws the masks of its own rows.
"""
import math
from functools import reduce

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32, "e4m3": torch.float8_e4m3fn}
SIZE = {"bf16": 2, "fp16": 2, "fp32": 4, "e4m3": 1}
EPS = 1e-6
MOST_8BIT = 448.0          # the largest value of e4m3


def listed():
    return [
        # a decoding step's residual and norm: nothing but latency
        {"name": "norm-1", "op": "norm", "n": 1, "dim": 4096, "dtype": "bf16", "sum": "bf16", "weight": "bf16", "out": "bf16", "residual": True, "drop": 0.0, "first": 0},
        # a prompt before projections in 8 bits, the residual kept in 32
        {"name": "norm-8bit-2000", "op": "norm", "n": 2000, "dim": 5120, "dtype": "bf16", "sum": "fp32", "weight": "fp32", "out": "e4m3", "residual": True, "drop": 0.0, "first": 0},
        # a training batch: dropout, residual and norm
        {"name": "norm-16384", "op": "norm", "n": 16384, "dim": 4096, "dtype": "bf16", "sum": "bf16", "weight": "bf16", "out": "bf16", "residual": True, "drop": 0.1, "first": 0},
        # a short fine-tuning batch, odd rows
        {"name": "norm-grad-257", "op": "norm_grad", "n": 257, "dim": 1001, "dtype": "fp16", "sum": "fp16", "weight": "fp32", "residual": True, "drop": 0.0, "first": 0},
        # the training batch's backward pass
        {"name": "norm-grad-16384", "op": "norm_grad", "n": 16384, "dim": 4096, "dtype": "bf16", "sum": "bf16", "weight": "bf16", "residual": True, "drop": 0.1, "first": 0},
        # embeddings of a short batch, a slice of a larger one
        {"name": "dropout-300", "op": "dropout", "n": 300, "dim": 1000, "dtype": "fp32", "drop": 0.25, "first": 300},
        # embeddings of a training batch
        {"name": "dropout-16384", "op": "dropout", "n": 16384, "dim": 4096, "dtype": "bf16", "drop": 0.1, "first": 0},
        # one token of a decoding step: the weights' bytes
        {"name": "gated-1", "op": "gated", "n": 1, "dim": 4096, "width": 12288, "dtype": "bf16", "act": "silu", "keep": False},
        # a prompt in 8 bits
        {"name": "gated-8bit-4096", "op": "gated", "n": 4096, "dim": 4096, "width": 12288, "dtype": "e4m3", "act": "silu", "keep": False},
        # a training batch, both projections kept for the gradient
        {"name": "gated-8192", "op": "gated", "n": 8192, "dim": 4096, "width": 12288, "dtype": "bf16", "act": "silu", "keep": True},
        # a short fine-tuning batch of a small model, odd sizes
        {"name": "gated-grad-200", "op": "gated_grad", "n": 200, "dim": 1000, "width": 2730, "dtype": "fp16", "act": "gelu"},
        # the training batch's backward pass
        {"name": "gated-grad-8192", "op": "gated_grad", "n": 8192, "dim": 4096, "width": 12288, "dtype": "bf16", "act": "silu"},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi):
    """Three in four are a multiple of 64, the others what they are."""
    v = _log(rng, lo, hi)
    return max(64, v // 64 * 64) if rng.random() < 0.75 else v


def draw(rng):
    op = rng.choice(["norm", "norm_grad", "dropout", "gated", "gated_grad"])
    if op.startswith("gated"):
        case = {"op": op, "n": _log(rng, 1, 8192), "dim": _size(rng, 64, 4096), "width": _size(rng, 64, 12288), "act": rng.choice(["silu", "silu", "gelu", "relu"])}
        case["dtype"] = rng.choice(["bf16", "bf16", "fp16"])
        if op == "gated":
            case["keep"] = rng.random() < 0.5
            if rng.random() < 0.3:
                case |= {"dtype": "e4m3", "keep": False}
        return case
    while True:
        n, dim = _log(rng, 1, 16384), _size(rng, 64, 16384)
        if n * dim <= 16384 * 4096:
            break
    dtype = rng.choice(["bf16", "bf16", "fp16", "fp32"])
    case = {"op": op, "n": n, "dim": dim, "dtype": dtype, "drop": rng.choice([0.1, 0.25, 0.5]), "first": rng.choice([0, 0, n])}
    if op != "dropout":
        case["drop"] = rng.choice([0.0, 0.0, case["drop"]])
        case |= {"sum": rng.choice([dtype, dtype, "fp32"]), "weight": rng.choice([dtype, "fp32"]), "residual": rng.random() < 0.8}
        if not case["residual"]:
            case["sum"] = dtype
        if op == "norm":
            case["out"] = rng.choice([dtype, dtype, "e4m3"])
    return case


def _to_8bit(x):
    """Rows in e4m3, each with a scale that takes its largest value to the type's."""
    scale = x.abs().amax(1) / MOST_8BIT
    return (x / scale[:, None]).to(torch.float8_e4m3fn), scale


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    n, dim, op = case["n"], case["dim"], case["op"]
    rand = lambda *shape: torch.randn(*shape, generator=g, device="cuda")  # noqa: E731
    state = {"case": case, "seed": 1000003 * seed + 17, "offset": ((seed & 0xFFFF) << 33) + 5}
    if op.startswith("gated"):
        width, dtype = case["width"], DTYPES[case["dtype"]]
        # normed rows, projections of unit variance
        x, weights = rand(n, dim), [rand(width, dim).mul_(dim ** -0.5) for _ in range(2)]
        if case["dtype"] == "e4m3":
            (state["x"], state["x_scale"]), (state["gate_weight"], state["gate_scale"]), (state["up_weight"], state["up_scale"]) = map(_to_8bit, [x] + weights)
            return state
        state |= {"x": x.to(dtype), "gate_weight": weights[0].to(dtype), "up_weight": weights[1].to(dtype)}
        if op == "gated_grad":
            state |= {"gate": (state["x"].float() @ state["gate_weight"].float().T).to(dtype), "up": (state["x"].float() @ state["up_weight"].float().T).to(dtype)}
            state["grad_out"] = rand(n, width).mul_(1e-2).to(dtype)
        return state
    dtype = DTYPES[case["dtype"]]
    # channels of different sizes, as a trained model's
    channel = (0.5 * rand(dim)).exp_()
    state["x"] = (rand(n, dim) * channel).to(dtype)
    if op == "dropout":
        return state
    state["weight"] = (1 + 0.2 * rand(dim)).to(DTYPES[case["weight"]])
    if case["residual"]:
        state["residual"] = (rand(n, dim) * 2 * channel).to(DTYPES[case["sum"]])
    if op == "norm_grad":
        # what the forward pass left: the sum and the rows' normalisers; gradients of the normed rows and of the sum
        state["total"] = state.pop("residual").add_(state["x"]) if case["residual"] else state["x"]
        state["rstd"] = (state["total"].float().square().mean(1) + EPS).rsqrt()
        state["grad_out"] = rand(n, dim).mul_(1e-2).to(dtype)
        if case["residual"]:
            state["grad_total"] = rand(n, dim).mul_(1e-2).to(DTYPES[case["sum"]])
        del state["x"]
    return state


# The generator: Philox 4x32 with 10 rounds (Salmon, Moraes, Dror, Shaw: "Parallel random numbers: as easy as 1, 2, 3", 2011).
# Counter: (columns by 8, row, offset); key: the seed.  Each of a counter's 8 numbers of 16 bits decides for one column.


def _round(state, _):
    a, b, c, d, k, q = state
    low = 0xFFFFFFFF
    # the upper half of a product of 32-bit numbers, whose 64 bits may wrap to negative ones
    ma, mc = a * 0xD2511F53, c * 0xCD9E8D57
    return (mc >> 32 & low) ^ b ^ k, mc & low, (ma >> 32 & low) ^ d ^ q, ma & low, (k + 0x9E3779B9) & low, (q + 0xBB67AE85) & low


def _kept(n, dim, drop, seed, offset, first, device):
    """1 / (share kept) where a value stays, 0 elsewhere."""
    units = -(-dim // 8)
    column = torch.arange(units, device=device)[None, :].expand(n, units)
    row = (torch.arange(n, device=device) + first)[:, None].expand(n, units)
    fill = lambda v: torch.full((1, 1), v & 0xFFFFFFFF, device=device)  # noqa: E731
    words = reduce(_round, range(10), (column, row, fill(offset), fill(offset >> 32), fill(seed), fill(seed >> 32)))[:4]
    bits = torch.stack([words[0] & 0xFFFF, words[0] >> 16, words[1] & 0xFFFF, words[1] >> 16,
                        words[2] & 0xFFFF, words[2] >> 16, words[3] & 0xFFFF, words[3] >> 16], -1).reshape(n, units * 8)[:, :dim]
    border = round(drop * 65536)
    return (bits >= border).float() * (65536 / (65536 - border))


def _plain_norm(s, case):
    total = s["x"].float()
    if case["drop"]:
        total = total * _kept(case["n"], case["dim"], case["drop"], s["seed"], s["offset"], case["first"], total.device)
    if case["residual"]:
        total = s["residual"].float() + total
    rstd = 1 / (total.square().mean(1) + EPS).sqrt()
    out, scale = total * rstd[:, None] * s["weight"].float(), None
    if case["out"] == "e4m3":
        scale = out.abs().amax(1) / MOST_8BIT
        out = out / scale[:, None]
    return out.to(DTYPES[case["out"]]), total.to(DTYPES[case["sum"]]) if case["residual"] or case["drop"] else None, rstd, scale


def _plain_norm_grad(s, case):
    normed, g = s["total"].float() * s["rstd"][:, None], s["grad_out"].float()
    grad_weight = (g * normed).sum(0)
    g = g * s["weight"].float()
    grad = (g - normed * (g * normed).mean(1, keepdim=True)) * s["rstd"][:, None]
    if case["residual"]:
        grad = grad + s["grad_total"].float()
    grad_x = grad
    if case["drop"]:
        grad_x = grad * _kept(case["n"], case["dim"], case["drop"], s["seed"], s["offset"], case["first"], grad.device)
    return grad_x.to(DTYPES[case["dtype"]]), grad.to(DTYPES[case["sum"]]) if case["residual"] else None, grad_weight.to(s["weight"].dtype)


def _plain_act(act, g):
    """(value, derivative)"""
    if act == "relu":
        return torch.where(g > 0, g, 0.0), (g > 0).float()
    # x * sigmoid(k(x)): the tanh form of gelu is one of these, too
    c = 2 * math.sqrt(2 / math.pi)
    k, dk = (g, 1.0) if act == "silu" else (c * (g + 0.044715 * g * g * g), c * (1 + 3 * 0.044715 * g * g))
    sigmoid = 1 / (1 + (-k).exp())
    return g * sigmoid, sigmoid + g * sigmoid * (1 - sigmoid) * dk


def _plain_gated(s, case):
    x, gate_weight, up_weight = s["x"].float(), s["gate_weight"].float(), s["up_weight"].float()
    gate, up = x @ gate_weight.T, x @ up_weight.T
    if case["dtype"] == "e4m3":
        gate, up = gate * s["x_scale"][:, None] * s["gate_scale"], up * s["x_scale"][:, None] * s["up_scale"]
    out = _plain_act(case["act"], gate)[0] * up
    dtype = torch.bfloat16 if case["dtype"] == "e4m3" else s["x"].dtype
    return (out.to(dtype), gate.to(dtype), up.to(dtype)) if case["keep"] else out.to(dtype)


def _plain_gated_grad(s, case):
    value, slope = _plain_act(case["act"], s["gate"].float())
    g, x = s["grad_out"].float(), s["x"].float()
    grad_gate, grad_up = g * s["up"].float() * slope, g * value
    dtype = s["x"].dtype
    return (grad_gate @ s["gate_weight"].float() + grad_up @ s["up_weight"].float()).to(dtype), (grad_gate.T @ x).to(dtype), (grad_up.T @ x).to(dtype)


def run(state):
    case, op = state["case"], state["case"]["op"]
    if own:
        import paper_1310_4645_b200 as rd
        if op == "norm":
            return rd.rd_norm(state["x"], state["weight"], state.get("residual"), eps=EPS, out_dtype=DTYPES[case["out"]], drop=case["drop"], seed=state["seed"],
                              offset=state["offset"], first_row=case["first"])
        if op == "norm_grad":
            return rd.rd_norm_grad(state["grad_out"], state["total"], state["weight"], state["rstd"], state.get("grad_total"), want_residual=case["residual"],
                                   drop=case["drop"], seed=state["seed"], offset=state["offset"], first_row=case["first"])
        if op == "dropout":
            return rd.rd_dropout(state["x"], case["drop"], state["seed"], state["offset"], first_row=case["first"])
        act = {"silu": rd.RD_SILU, "gelu": rd.RD_GELU, "relu": rd.RD_RELU}[case["act"]]
        if op == "gated":
            out, gate, up = rd.rd_gated(state["x"], state["gate_weight"], state["up_weight"], activation=act, keep=case["keep"], x_scale=state.get("x_scale"),
                                        gate_scale=state.get("gate_scale"), up_scale=state.get("up_scale"))
            return (out, gate, up) if case["keep"] else out
        return rd.rd_gated_grad(state["grad_out"], state["x"], state["gate_weight"], state["up_weight"], state["gate"], state["up"], activation=act)
    if op == "norm":
        return _plain_norm(state, case)
    if op == "norm_grad":
        return _plain_norm_grad(state, case)
    if op == "dropout":
        x = state["x"]
        return (x.float() * _kept(case["n"], case["dim"], case["drop"], state["seed"], state["offset"], case["first"], x.device)).to(x.dtype)
    return _plain_gated(state, case) if op == "gated" else _plain_gated_grad(state, case)


def work(case):
    n, dim, op, size = case["n"], case["dim"], case["op"], SIZE[case["dtype"]]
    if op == "dropout":
        return {"bytes": 2 * n * dim * size, "flops": n * dim}
    if op.startswith("norm"):
        sums, weight = SIZE[case["sum"]], dim * SIZE[case["weight"]]
        if op == "norm":
            stored = case["residual"] or case["drop"] > 0
            return {"bytes": n * dim * (size + (sums if case["residual"] else 0) + (sums if stored else 0) + SIZE[case["out"]]) + weight + 4 * n * (2 if case["out"] == "e4m3" else 1),
                    "flops": 6 * n * dim}
        # without dropout, in one type, the gradients of the residual and of x are the same matrix
        both = case["residual"] and (case["drop"] > 0 or case["sum"] != case["dtype"])
        return {"bytes": n * dim * (2 * size + sums + (sums if case["residual"] else 0) + (sums if both else 0)) + 2 * weight + 4 * n, "flops": 10 * n * dim}
    width = case["width"]
    if op == "gated":
        out = 2 * n * width * (3 if case["keep"] else 1)
        return {"bytes": (n + 2 * width) * dim * size + out, "flops": 4 * n * dim * width}
    return {"bytes": (3 * n * width + 2 * n * dim + 4 * width * dim) * size, "flops": 8 * n * dim * width}


def _exact_kept(case, s):
    """The generator by halves of 16 bits, so that no product passes 32."""
    n, dim = case["n"], case["dim"]
    device = "cuda"

    def product(c, m):
        """(upper, lower) 32 bits of c * m"""
        c0, c1, m0, m1 = c & 0xFFFF, c >> 16, m & 0xFFFF, m >> 16
        middle = c1 * m0 + (c0 * m0 >> 16)
        cross = c0 * m1 + (middle & 0xFFFF)
        return c1 * m1 + (middle >> 16) + (cross >> 16), (cross & 0xFFFF) << 16 | (c0 * m0 & 0xFFFF)

    j = torch.arange(dim, device=device)
    r = torch.arange(n, device=device)[:, None] + case["first"]
    counter = [(j // 8).unique()[None, :] + 0 * r, r + 0 * (j // 8).unique()[None, :], s["offset"] % 2 ** 32 + 0 * r, s["offset"] // 2 ** 32 + 0 * r]
    for turn in range(10):
        k0, k1 = (s["seed"] % 2 ** 32 + turn * 0x9E3779B9) % 2 ** 32, (s["seed"] // 2 ** 32 + turn * 0xBB67AE85) % 2 ** 32
        (h0, l0), (h1, l1) = product(counter[0], 0xD2511F53), product(counter[2], 0xCD9E8D57)
        counter = [h1 ^ counter[1] ^ k0, l1, h0 ^ counter[3] ^ k1, l0]
    words = torch.stack(counter, -1)                                   # [n, units, 4]
    number = words[:, j // 8, j % 8 // 2] // torch.where(j % 2 == 1, 65536, 1) % 65536
    border = int(round(case["drop"] * 65536))
    return torch.where(number < border, 0.0, 65536.0 / (65536.0 - border)).double()


def exact(case, seed):
    """The definitions in 64 bits, element by element."""
    s = prepare(case, seed)
    op = case["op"]
    if op == "dropout":
        return s["x"].double().mul(_exact_kept(case, s))
    if op == "norm":
        total = s["x"].double()
        if case["drop"] > 0:
            total.mul_(_exact_kept(case, s))
        if case["residual"]:
            total.add_(s["residual"].double())
        length = torch.sqrt(torch.linalg.vector_norm(total, dim=1).square().div(case["dim"]).add(EPS))
        out = torch.div(total, length[:, None]).mul_(s["weight"].double()[None, :])
        scale = None
        if case["out"] == "e4m3":
            scale = torch.linalg.vector_norm(out, ord=math.inf, dim=1).div(MOST_8BIT)
            out.div_(scale[:, None])
        return out, total if case["residual"] or case["drop"] > 0 else None, length.reciprocal(), scale
    if op == "norm_grad":
        total, up, r = s["total"].double(), s["grad_out"].double(), s["rstd"].double()
        # d/ds of  sum_j up_j w_j s_j r(s),  r' = -r^3 s / dim
        scaled = up * s["weight"].double()[None, :]
        dot = torch.linalg.vecdot(scaled, total)
        grad = scaled.mul(r[:, None]).sub_(total.mul((dot * r.pow(3) / case["dim"])[:, None]))
        grad_weight = torch.einsum("ij,ij,i->j", up, total, r)
        if case["residual"]:
            grad.add_(s["grad_total"].double())
        return grad.mul(_exact_kept(case, s)) if case["drop"] > 0 else grad, grad if case["residual"] else None, grad_weight
    if op == "gated":
        x = s["x"].double()
        gate, up = torch.mm(x, s["gate_weight"].double().t()), torch.mm(x, s["up_weight"].double().t())
        if case["dtype"] == "e4m3":
            gate.mul_(torch.outer(s["x_scale"].double(), s["gate_scale"].double()))
            up.mul_(torch.outer(s["x_scale"].double(), s["up_scale"].double()))
        out = {"silu": torch.nn.functional.silu, "relu": torch.relu, "gelu": lambda v: torch.nn.functional.gelu(v, approximate="tanh")}[case["act"]](gate).mul_(up)
        return (out, gate, up) if case["keep"] else out
    gate, up, g = s["gate"].double(), s["up"].double(), s["grad_out"].double()
    if case["act"] == "silu":
        sigma = torch.sigmoid(gate)
        value, slope = gate * sigma, sigma.mul(1 + gate - gate * sigma)
    elif case["act"] == "gelu":
        root = math.sqrt(2 / math.pi)
        t = torch.tanh(root * gate * (1 + 0.044715 * gate.square()))
        value = 0.5 * gate * (1 + t)
        slope = 0.5 * (1 + t) + 0.5 * gate * (1 - t.square()) * root * (1 + 0.134145 * gate.square())
    else:
        value, slope = gate.clamp(min=0), gate.gt(0).double()
    d_gate, d_up = slope.mul_(up).mul_(g), value.mul_(g)
    x = s["x"].double()
    return torch.addmm(torch.mm(d_gate, s["gate_weight"].double()), d_up, s["up_weight"].double()), torch.mm(d_gate.t(), x), torch.mm(d_up.t(), x)
