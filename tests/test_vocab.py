"""Embedding lookup, softmax cross entropy over a vocabulary and their gradients, against their definitions in 64 bits.

Bounds.  u is the unit round-off of the result's type (bf16 2^-8, fp16 2^-11, fp32 2^-24).  A fp32 sum of c terms is off by at
most c * 2^-23 times the sum of their magnitudes (2^-23 per addition also where an adder truncates).  A logit is such a sum of dim
exact products, off by dx; lse and a probability inherit dx (lse absolutely, a probability relatively), and an exponential or
logarithm adds 2^-20 at the magnitudes that occur.  dx of the gradient is rounded to 16 bits once: u relatively.
"""
import ctypes as C
import math

import pytest
import torch

import paper_1310_4645_b200 as rd

gpu = pytest.mark.gpu
U = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24}      # spacing of the subnormal numbers
HALF = [torch.bfloat16, torch.float16]


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def rand(*shape, seed=0, dtype=torch.float32, std=1.0):
    return torch.randn(*shape, generator=gen(seed), device="cuda").mul_(std).to(dtype)


def ints(lo, hi, n, seed=0, dtype=torch.int64):
    return torch.randint(lo, hi, (n,), generator=gen(seed), device="cuda").to(dtype)


def strided(t, pad, offset=0):
    """The same values with `pad` extra elements per row, beginning `offset` elements into an allocation."""
    rows, dim = t.shape
    big = torch.full((rows * (dim + pad) + offset,), float("nan"), dtype=t.dtype, device=t.device)
    view = big[offset:].view(rows, dim + pad)[:, :dim]
    view.copy_(t)
    return view


def within(got, want, bound):
    got = got.double()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    off = torch.where(torch.isnan(want), 0.0, (got - want).abs())
    worst = (off - bound).max().item() if off.numel() else -1.0
    assert worst <= 0, "off by %.3g more than the bound; largest error %.3g" % (worst, off.max().item())


# ------------------------------------------------------------------------------------------------ embedding


@gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("n, rows, dim, pad, offset", [(1, 7, 8, 0, 0), (1, 1, 1, 0, 0), (5, 3, 1, 2, 1), (33, 100, 64, 8, 0), (257, 61, 129, 0, 0),
                                                       (64, 1000, 1000, 0, 8), (1000, 50, 100, 4, 3), (300, 20, 2056, 0, 0)])
def test_embed(dtype, n, rows, dim, pad, offset):
    table = strided(rand(rows, dim, seed=1, dtype=dtype), pad, offset)
    ids = ints(-2, rows + 3, n, seed=2, dtype=torch.int32 if n % 2 else torch.int64)
    inside = (ids >= 0) & (ids < rows)
    for scale in (1.0, -math.sqrt(dim)):
        want = torch.zeros(n, dim, dtype=torch.float64, device="cuda")
        want[inside] = table.double()[ids[inside].long()] * torch.tensor(scale).double().item()
        out = strided(torch.zeros(n, dim, dtype=dtype, device="cuda"), pad, offset)
        assert rd.rd_embed(table, ids, out, scale=scale) is out
        bound = 0.0 if scale == 1.0 else (U[dtype] + 2.0 ** -23) * want.abs() + TINY[dtype]
        within(out, want, torch.as_tensor(bound, device="cuda"))
        assert torch.equal(rd.rd_embed(table, ids, scale=scale), out)


@gpu
def test_embed_slices_add_up():
    """Every id is found in exactly one of the slices, the others give zeros; ids far outside stay outside."""
    table, ids = rand(96, 40, seed=3), ints(0, 96, 200, seed=4)
    parts = [rd.rd_embed(table[a:b], ids, first_row=a) for a, b in ((0, 32), (32, 33), (33, 96))]
    assert torch.equal(sum(parts), table[ids])
    far = torch.tensor([2 ** 62, -2 ** 63, 2 ** 40 + 5, 2 ** 31, 95 + 2 ** 32], device="cuda")
    assert not rd.rd_embed(table, far).any()
    assert torch.equal(rd.rd_embed(table, far, first_row=2 ** 40)[2], table[5])


def grad_reference(grad, ids, rows, first, scale, base=None):
    at = ids.long() - first
    keep = (ids >= 0) & (at >= 0) & (at < rows)
    total = torch.zeros(rows, grad.shape[1], dtype=torch.float64, device="cuda")
    size = torch.zeros_like(total)
    total.index_add_(0, at[keep], grad[keep].double())
    size.index_add_(0, at[keep], grad[keep].double().abs())
    count = torch.bincount(at[keep], minlength=rows).double()[:, None]
    want = total * scale
    bound = (count + 2) * 2.0 ** -23 * size * abs(scale)
    if base is not None:
        want, bound = want + base.double(), bound + 2.0 ** -23 * (base.double().abs() + want.abs())
    return want, bound, count[:, 0] > 0


@gpu
@pytest.mark.parametrize("dtype, out", [(torch.float32, torch.float32), (torch.bfloat16, torch.bfloat16), (torch.bfloat16, torch.float32),
                                        (torch.float16, torch.float16), (torch.float16, torch.float32)])
@pytest.mark.parametrize("n, rows, dim, pad, ids", [(1, 5, 8, 0, "uniform"), (3, 1, 1, 0, "uniform"), (500, 37, 24, 0, "uniform"), (64, 9, 65, 1, "same"),
                                                    (65, 9, 64, 0, "same"), (1000, 3000, 520, 8, "skewed"), (4096, 3, 48, 0, "skewed"), (4097, 900, 64, 16, "uniform"), (9001, 1025, 40, 0, "skewed"),
                                                    (70000, 2050, 8, 0, "skewed"), (300000, 11, 4, 0, "same"), (20000, 3, 520, 0, "same"), (5000, 70, 1032, 8, "skewed"), (50, 40, 33, 0, "outside")])
@pytest.mark.parametrize("accumulate", [False, True])
def test_embed_grad(dtype, out, n, rows, dim, pad, ids, accumulate):
    grad = strided(rand(n, dim, seed=5, dtype=dtype), pad)
    first = 1000
    at = {"uniform": lambda: ints(-3, rows + 3, n, seed=6), "same": lambda: torch.full((n,), rows // 2, device="cuda"),
          "skewed": lambda: (torch.exp(torch.rand(n, generator=gen(7), device="cuda") * math.log(rows + 1)).long() - 1),
          "outside": lambda: ints(rows, rows + 9, n, seed=8)}[ids]()
    tokens = (at + first).to(torch.int64 if n % 2 else torch.int32)
    base = rand(rows, dim, seed=9, dtype=out)
    table = strided(base, pad)
    want, bound, touched = grad_reference(grad, tokens, rows, first, 0.75, base if accumulate else None)
    rd.rd_embed_grad(grad, tokens, table, first_row=first, scale=0.75, accumulate=accumulate)
    within(table, want, bound + U[out] * want.abs() + TINY[out])
    if accumulate:
        assert torch.equal(table[~touched], base[~touched])
    # the same bits every time, whatever order the atomics took, and in a workspace full of something else
    again = strided(base, pad)
    ws = torch.full((rd.rd_embed_grad_workspace(rows, dim, n),), 255, dtype=torch.uint8, device="cuda")
    rd.rd_embed_grad(grad, tokens, again, first_row=first, scale=0.75, accumulate=accumulate, workspace=ws)
    assert torch.equal(table, again)


@gpu
@pytest.mark.parametrize("dtype, out, n, rows, dim, pad", [(torch.bfloat16, torch.bfloat16, 9001, 401003, 264, 0), (torch.bfloat16, torch.float32, 30000, 110007, 512, 0),
                                                           (torch.float32, torch.float32, 5001, 100001, 516, 8), (torch.float16, torch.float16, 70000, 20011, 8192, 0),
                                                           (torch.bfloat16, torch.bfloat16, 6000, 300001, 40, 600)])
def test_embed_grad_large_tables(dtype, out, n, rows, dim, pad):
    """Tables that are filled in two parts, the second beside the sums: on two streams at once, and recorded into a graph as well."""
    grad, tokens = rand(n, dim, seed=30, dtype=dtype), (torch.exp(torch.rand(n, generator=gen(31), device="cuda") * math.log(rows + 1)).long() - 1).flip(0)
    tokens = torch.where(tokens % 2 == 0, tokens, rows - 1 - tokens)      # frequent rows in both parts
    fresh = lambda: strided(torch.full((rows, dim), 7.0, dtype=out, device="cuda"), pad)
    want, bound, touched = grad_reference(grad, tokens, rows, 0, 1.25)
    table = rd.rd_embed_grad(grad, tokens, fresh(), scale=1.25)
    within(table, want, bound + U[out] * want.abs() + TINY[out])
    assert not table[~touched].any()
    del want, bound
    streams, tables = [torch.cuda.Stream() for _ in range(2)], [fresh() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(3):
        for s, t in zip(streams, tables):
            with torch.cuda.stream(s):
                t.fill_(7.0)
                rd.rd_embed_grad(grad, tokens, t, scale=1.25)
    torch.cuda.synchronize()
    assert all(torch.equal(t, table) for t in tables)
    graph, ws = torch.cuda.CUDAGraph(), torch.empty(rd.rd_embed_grad_workspace(rows, dim, n), dtype=torch.uint8, device="cuda")
    with torch.cuda.graph(graph):
        rd.rd_embed_grad(grad, tokens, tables[0], scale=1.25, workspace=ws)
    tables[0].fill_(7.0)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(tables[0], table) and rd.rd_vocab_status() == rd.RD_OK


@gpu
def test_embed_grad_is_the_derivative():
    """The lookup is linear, so a difference quotient of <grad, lookup(table)> is the gradient's entry up to rounding."""
    table, ids, grad = rand(11, 6, seed=10), ints(0, 11, 40, seed=11), rand(40, 6, seed=12)
    g = rd.rd_embed_grad(grad, ids, torch.empty_like(table), scale=3.0)
    for v, j in ((0, 0), (4, 5), (10, 2)):
        moved = table.clone()
        moved[v, j] += 1.0
        diff = ((rd.rd_embed(moved, ids, scale=3.0).double() - rd.rd_embed(table, ids, scale=3.0).double()) * grad.double()).sum().item()
        # 40 lookups of magnitude < 16, each rounded by 2^-24 twice
        assert abs(diff - g[v, j].item()) <= 40 * 2 * 16 * 2.0 ** -24 * grad.abs().max().item() * 2


@gpu
def test_embed_grad_special_values():
    """Tokens outside the slice contribute nothing whatever they hold; a broadcast gradient row; no tokens."""
    ids = torch.tensor([0, 7, -1, 1, 0], device="cuda")
    grad = rand(5, 16, seed=13)
    grad[1] = float("nan")
    grad[2] = float("inf")
    g = rd.rd_embed_grad(grad, ids, torch.empty(3, 16, device="cuda"))
    assert torch.equal(g[0], grad[0] + grad[4]) and torch.equal(g[1], grad[3]) and not g[2].any()
    g = rd.rd_embed_grad(grad[:1].expand(5, 16), ids, torch.empty(3, 16, device="cuda"))
    assert torch.equal(g[0], grad[0] * 2) and torch.equal(g[1], grad[0])
    g = rd.rd_embed_grad(grad[:0], ids[:0], torch.full((3, 16), 5.0, device="cuda"))
    assert not g.any()
    g = rd.rd_embed_grad(grad[:0], ids[:0], torch.full((3, 16), 5.0, device="cuda"), accumulate=True)
    assert (g == 5).all()


# ------------------------------------------------------------------------------------------------ loss


def loss_reference(hidden, weight, labels, first, scale, z):
    """(loss, lse, target, logits, bound of a logit's error) in 64 bits."""
    h, w = hidden.double(), weight.double()
    counts = labels >= 0
    h = torch.where(counts[:, None], h, 0.0)
    x = h @ w.T * scale
    err = (h.abs() @ w.abs().T) * abs(scale) * (hidden.shape[1] + 4) * 2.0 ** -23
    at = labels.long() - first
    here = counts & (at >= 0) & (at < weight.shape[0])
    lse = torch.where(counts, torch.logsumexp(x, 1), 0.0)
    target = torch.where(here, x.gather(1, torch.where(here, at, 0)[:, None])[:, 0], 0.0)
    loss = torch.where(counts, lse - target + z * lse * lse, 0.0)
    return loss, lse, target, x, err, here, torch.where(here, at, 0)


SHAPES = [(1, 1, 1), (3, 1000, 4096), (4, 777, 1001), (4, 70000, 40), (1, 33, 16400), (9, 100, 72), (64, 9000, 128), (100, 20000, 40), (1, 300, 64), (2, 5, 3), (37, 257, 72), (128, 256, 64), (129, 511, 65), (300, 1000, 200), (513, 77, 1032), (40, 5000, 33), (1, 32768, 128)]


def vocab_case(n, rows, dim, dtype, seed, ignored=0.25, first=0, label_dtype=torch.int64):
    weight = rand(rows, dim, seed=seed, dtype=dtype, std=2.0 / math.sqrt(dim))
    hidden = rand(n, dim, seed=seed + 1, dtype=dtype)
    labels = ints(0, rows, n, seed=seed + 2) + first
    if n > 2:
        drop = torch.rand(n, generator=gen(seed + 3), device="cuda") < ignored
        labels[drop] = -100
    return hidden, weight, labels.to(label_dtype)


def check_loss(hidden, weight, labels, first=0, scale=1.0, z=0.0):
    loss, lse, target = rd.rd_vocab_loss(hidden, weight, labels, first_row=first, scale=scale, z_loss=z)
    wl, wn, wt, x, err, here, at = loss_reference(hidden, weight, labels, first, scale, z)
    e = err.amax(1)
    counts = (labels >= 0).double()
    bn = (e + 2.0 ** -20 + 2.0 ** -22 * (wn.abs() + x.abs().amax(1))) * counts
    bt = (e + 2.0 ** -23 * wt.abs()) * counts
    within(lse, wn, bn)
    within(target, wt, bt)
    within(loss, wl, bn * (1 + 2 * abs(z) * wn.abs()) + bt + 2.0 ** -22 * (wl.abs() + wn.abs() + wt.abs() + abs(z) * wn * wn))
    assert rd.rd_vocab_status() == rd.RD_OK
    return loss, lse, target


@gpu
@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("n, rows, dim", SHAPES)
def test_loss(dtype, n, rows, dim):
    hidden, weight, labels = vocab_case(n, rows, dim, dtype, seed=20, label_dtype=torch.int32 if rows % 2 else torch.int64)
    check_loss(hidden, weight, labels, scale=0.7, z=1e-2)
    # rows that are not aligned to 16 bytes, and ones with a stride
    check_loss(strided(hidden, 3, 1), strided(weight, 1, 3), labels)
    check_loss(strided(hidden, 8), strided(weight, 16), labels, scale=-1.5)


@gpu
@pytest.mark.parametrize("dtype", HALF)
def test_loss_slices_join(dtype):
    """lse and target of slices, joined, are the whole vocabulary's."""
    hidden, weight, labels = vocab_case(70, 1100, 96, dtype, seed=30)
    loss, lse, target = check_loss(hidden, weight, labels)
    parts = [rd.rd_vocab_loss(hidden, weight[a:b], labels, first_row=a) for a, b in ((0, 300), (300, 301), (301, 1100))]
    counts = labels >= 0
    joined = torch.where(counts, torch.logsumexp(torch.stack([p[1] for p in parts]), 0), 0.0)
    assert torch.allclose(joined, lse, rtol=0, atol=1e-5)
    assert torch.equal(sum(p[2] for p in parts), target)


@gpu
def test_loss_special_values():
    """Ignored rows may hold anything; infinite logits give infinite lse, NaN a NaN, in their own row only."""
    hidden, weight, labels = vocab_case(200, 600, 64, torch.bfloat16, seed=40, ignored=0.0)
    labels[::3] = -1
    clean = check_loss(hidden, weight, labels)
    dirty = hidden.clone()
    dirty[::3] = float("nan")
    dirty[3] = float("inf")
    for a, b in zip(clean, rd.rd_vocab_loss(dirty, weight, labels)):
        assert torch.equal(a, b)
    dirty[1] = float("nan")
    loss, lse, _ = rd.rd_vocab_loss(dirty, weight, labels)
    assert torch.isnan(lse[1]) and torch.isnan(loss[1])
    rest = torch.arange(200, device="cuda") != 1
    assert torch.equal(lse[rest], clean[1][rest]) and torch.equal(loss[rest], clean[0][rest])


@gpu
@pytest.mark.parametrize("n", [2, 20])
def test_loss_infinite_logits(n):
    # hidden e_0, weight rows 0 except a +-infinite one
    h = torch.zeros(n, 8, dtype=torch.bfloat16, device="cuda")
    h[:, 0] = 1
    w = torch.zeros(300, 8, dtype=torch.bfloat16, device="cuda")
    w[299, 0] = float("-inf")
    lab = torch.arange(n, device="cuda") + 3
    loss, lse, target = rd.rd_vocab_loss(h, w, lab)
    assert torch.allclose(lse, torch.full_like(lse, math.log(299)), rtol=1e-6)
    w[280, 0] = float("inf")
    loss, lse, target = rd.rd_vocab_loss(h, w, lab)
    assert torch.isposinf(lse).all() and torch.isposinf(loss).all() and not target.any()
    # every logit is the lowest: nothing to normalise
    w[:, 0] = float("-inf")
    assert torch.isneginf(rd.rd_vocab_loss(h, w, lab)[1]).all()
    # very low and very high finite logits
    w[:, 0] = -30000.0
    assert torch.allclose(rd.rd_vocab_loss(h, w, lab)[1].double().cpu(), torch.full((n,), w[0, 0].double().item() + math.log(300), dtype=torch.float64), rtol=1e-6)
    # tokens that do not count, whatever they hold
    lab[1] = -1
    h[1] = float("nan")
    loss, lse, target = rd.rd_vocab_loss(h, w, lab)
    assert loss[1] == 0 and lse[1] == 0 and target[1] == 0 and torch.isfinite(lse).all()
    lab[:] = -100
    assert not any(t.any() for t in rd.rd_vocab_loss(h, w, lab))
    assert all(t.numel() == 0 for t in rd.rd_vocab_loss(h[:0], w, lab[:0]))


# ------------------------------------------------------------------------------------------------ gradient of the loss


def check_grad(hidden, weight, labels, up, first=0, scale=1.0, z=0.0, shift=0.0, pad=0, offset=0):
    dtype, (n, dim), rows = hidden.dtype, hidden.shape, weight.shape[0]
    _, lse64, _, x, err, here, at = loss_reference(hidden, weight, labels, first, scale, z)
    lse = (lse64 + shift).float()                       # shift: the part of the normaliser that other slices hold
    gh = strided(torch.full((n, dim), 7.0, dtype=dtype, device="cuda"), pad, offset)
    gw = strided(torch.full((rows, dim), 7.0, dtype=dtype, device="cuda"), pad, offset)
    rd.rd_vocab_loss_grad(hidden, weight, labels, lse, up, gh, gw, first_row=first, scale=scale, z_loss=z)
    counts = labels >= 0
    g = torch.where(counts, up.double(), 0.0)
    n64 = lse.double()
    h = torch.where(counts[:, None], hidden.double(), 0.0)
    w = weight.double()
    p = (x - n64[:, None]).exp() * (g * (1 + 2 * z * n64))[:, None]
    one = torch.zeros_like(p)
    one[torch.arange(n, device="cuda")[here], at[here]] = g[here]
    dx = (p - one) * scale
    # relative error of p: the logit's, the exponential's, the factors'; then one rounding to 16 bits, for fp16 also in units of its
    # smallest number after the largest factor was moved to at least 2^13
    d = (p.abs() * (err + 2.0 ** -20 + 2.0 ** -22 * (x.abs() + n64.abs()[:, None])) + 2.0 ** -22 * one.abs()) * abs(scale)
    d = d + U[dtype] * (dx.abs() + d)
    if dtype == torch.float16:
        d = d + 2.0 ** -25 * 2.0 ** -13 * 2 * torch.maximum(g.abs().max(), (g * (1 + 2 * z * n64)).abs().max()) * abs(scale)
    d = d * counts[:, None]
    for got, want, size, bound in ((gh, dx @ w, dx.abs() @ w.abs(), d @ w.abs()), (gw, dx.T @ h, dx.abs().T @ h.abs(), d.T @ h.abs())):
        terms = rows if want.shape[0] == n else n
        bound = bound + (terms + 8) * 2.0 ** -23 * (size + bound)
        within(got, want, bound + U[dtype] * (want.abs() + bound) + TINY[dtype])
    assert rd.rd_vocab_status() == rd.RD_OK
    # bit for bit the same again, each gradient alone, in a workspace full of something else
    ws = torch.full((rd.rd_vocab_loss_grad_workspace(hidden, weight, labels, True, True),), 255, dtype=torch.uint8, device="cuda")
    alone_h, alone_w = torch.empty_like(gh), torch.empty_like(gw)
    rd.rd_vocab_loss_grad(hidden, weight, labels, lse, up, alone_h, None, first_row=first, scale=scale, z_loss=z, workspace=ws)
    rd.rd_vocab_loss_grad(hidden, weight, labels, lse, up, None, alone_w, first_row=first, scale=scale, z_loss=z, workspace=ws)
    assert torch.equal(alone_h, gh) and torch.equal(alone_w, gw)
    return gh, gw


@gpu
@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("n, rows, dim", SHAPES)
def test_loss_grad(dtype, n, rows, dim):
    hidden, weight, labels = vocab_case(n, rows, dim, dtype, seed=50, label_dtype=torch.int32 if rows % 2 else torch.int64)
    up = (0.5 + torch.rand(n, generator=gen(51), device="cuda")) / n
    check_grad(hidden, weight, labels, up, scale=0.7, z=1e-2)
    check_grad(strided(hidden, 3, 1), strided(weight, 1, 3), labels, up, pad=5, offset=1)
    check_grad(strided(hidden, 8), strided(weight, 16), labels, torch.full((), 1.0 / n, device="cuda").expand(n), scale=-1.5, pad=8)


@gpu
@pytest.mark.parametrize("dtype", HALF)
def test_loss_grad_of_a_slice(dtype):
    hidden, weight, labels = vocab_case(150, 700, 80, dtype, seed=60)
    up = torch.full((150,), 1e-3, device="cuda")
    labels = torch.where(labels % 2 == 1, labels + 700, labels)      # odd ones: labels of the other slice
    check_grad(hidden, weight, labels, up, shift=0.7)
    labels = torch.where(labels >= 0, labels + 5000, labels)
    check_grad(hidden, weight, labels, up, first=5000, shift=0.7)


@gpu
@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("size", [1e-9, 1.0, 1e3])
def test_loss_grad_sizes_of_the_upstream_gradient(dtype, size):
    """fp16: probabilities times a small gradient would vanish without the power of two."""
    hidden, weight, labels = vocab_case(40, 2000, 64, dtype, seed=70)
    up = torch.full((40,), size, device="cuda")
    up[3] = 0.0
    check_grad(hidden, weight, labels, up)


@gpu
def test_loss_grad_pieces():
    """More tokens than one piece of the vocabulary, or one band of statistics, has room for."""
    hidden, weight, labels = vocab_case(40000, 9000, 64, torch.bfloat16, seed=80)
    check_loss(hidden[:, :64], weight[:1500], labels % 1500)            # and several bands of tokens in the loss
    check_grad(hidden, weight, labels, torch.full((40000,), 1.0 / 30000, device="cuda"))


@gpu
@pytest.mark.parametrize("dtype", HALF)
def test_loss_grad_special_values(dtype):
    hidden, weight, labels = vocab_case(200, 600, 64, dtype, seed=90, ignored=0.0)
    up = torch.full((200,), 1.0 / 200, device="cuda")
    labels[::3] = -1
    gh, gw = check_grad(hidden, weight, labels, up)
    assert not gh[::3].any()
    _, lse, _ = rd.rd_vocab_loss(hidden, weight, labels)
    ref = rd.rd_vocab_loss_grad(hidden, weight, labels, lse, up, torch.empty_like(hidden), torch.empty_like(weight))
    dirty, dirty_lse, dirty_up = hidden.clone(), lse.clone(), up.clone()
    dirty[::3] = float("nan")
    dirty_lse[::3] = float("inf")
    dirty_up[::3] = float("nan")
    got = rd.rd_vocab_loss_grad(dirty, weight, labels, dirty_lse, dirty_up, torch.empty_like(hidden), torch.empty_like(weight))
    assert torch.equal(got[0], ref[0]) and torch.equal(got[1], ref[1])
    # nothing counts, no tokens
    labels[:] = -100
    gh, gw = rd.rd_vocab_loss_grad(dirty, weight, labels, dirty_lse, dirty_up, torch.ones_like(hidden), torch.ones_like(weight))
    assert not gh.any() and not gw.any()
    gh, gw = rd.rd_vocab_loss_grad(hidden[:0], weight, labels[:0], lse[:0], up[:0], torch.empty_like(hidden[:0]), torch.ones_like(weight))
    assert not gw.any()


@gpu
def test_loss_grad_is_the_derivative():
    """Central differences of the summed loss along a random direction, of hidden and of weight."""
    hidden, weight, labels = vocab_case(24, 90, 16, torch.float16, seed=100)
    n = 24
    up = torch.linspace(0.5, 1.5, n, device="cuda")

    def total(h, w):                                       # the definition, in 64 bits
        x = h @ w.T * 0.9
        lse = torch.logsumexp(x, 1)
        t = x.gather(1, labels.clamp(min=0)[:, None])[:, 0]
        return (torch.where(labels >= 0, lse - t + 1e-2 * lse * lse, 0.0) * up.double()).sum()

    h, w = hidden.double(), weight.double()
    _, lse, _ = rd.rd_vocab_loss(hidden, weight, labels, scale=0.9, z_loss=1e-2)
    gh, gw = rd.rd_vocab_loss_grad(hidden, weight, labels, lse, up, torch.empty_like(hidden), torch.empty_like(weight), scale=0.9, z_loss=1e-2)
    for g, at, f in ((gh, h, lambda d: total(h + d, w)), (gw, w, lambda d: total(h, w + d))):
        direction = rand(*at.shape, seed=101).double()
        eps = 1e-5
        diff = ((f(eps * direction) - f(-eps * direction)) / (2 * eps)).item()
        along = (g.double() * direction).sum().item()
        # every entry carries two roundings of 2^-11 (dx, result); entries of dx cancel in the sums that make up g by a factor
        # of at most the sum of their magnitudes over g, below 8 in norm here
        assert abs(diff - along) <= 16 * 2.0 ** -11 * (g.double().norm() * direction.norm()).item()


@gpu
def test_streams_and_graphs():
    """Calls follow their stream, and replay from a CUDA graph on new values."""
    hidden, weight, labels = vocab_case(100, 900, 64, torch.bfloat16, seed=110)
    up = torch.full((100,), 0.01, device="cuda")
    want = rd.rd_vocab_loss(hidden, weight, labels)
    want_g = rd.rd_vocab_loss_grad(hidden, weight, labels, want[1], up, torch.empty_like(hidden), torch.empty_like(weight))
    want_e = rd.rd_embed(weight, labels, scale=2.0)
    want_t = rd.rd_embed_grad(hidden, labels, torch.empty_like(weight))
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    h = torch.zeros_like(hidden)
    gh, gw, e, t = torch.empty_like(hidden), torch.empty_like(weight), torch.empty_like(hidden), torch.empty_like(weight)

    def calls():
        out = rd.rd_vocab_loss(h, weight, labels)
        rd.rd_vocab_loss_grad(h, weight, labels, out[1], up, gh, gw)
        rd.rd_embed(weight, labels, e, scale=2.0)
        rd.rd_embed_grad(h, labels, t)
        return out

    with torch.cuda.stream(side):
        h.copy_(hidden, non_blocking=True)
        out = calls()
    side.synchronize()
    for a, b in zip((*out, gh, gw, e, t), (*want, *want_g, want_e, want_t)):
        assert torch.equal(a, b)
    h.zero_()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = calls()
    h.copy_(hidden)
    graph.replay()
    torch.cuda.synchronize()
    for a, b in zip((*out, gh, gw, e, t), (*want, *want_g, want_e, want_t)):
        assert torch.equal(a, b)
    out = rd.rd_vocab_loss(hidden, weight, labels, stream=side)
    e2 = rd.rd_embed(weight, labels, scale=2.0, stream=side)
    side.synchronize()
    assert torch.equal(out[0], want[0]) and torch.equal(e2, want_e)


# ------------------------------------------------------------------------------------------------ refusals (no GPU needed)


P = 1 << 20      # stands for device addresses: refused calls touch none


def test_embed_refusals():
    L = rd.lib()

    def call(table=P, tstride=8, rows=16, dim=8, dtype=rd.RD_BF16, ids=4 * P, idt=rd.RD_INT64, n=4, first=0, scale=1.0, out=2 * P, ostride=8):
        return L.rd_embed(table, tstride, rows, dim, dtype, ids, idt, n, first, scale, out, ostride, None)

    bad = rd.RD_ERR_INVALID_ARG
    assert call(n=0) == rd.RD_OK
    for kw in (dict(table=None), dict(ids=None), dict(out=None), dict(table=P + 1), dict(ids=4 * P + 4), dict(out=2 * P + 1), dict(tstride=7), dict(ostride=7), dict(ostride=0),
               dict(tstride=0), dict(rows=0), dict(dim=0), dict(dim=65537, tstride=65537, ostride=65537), dict(dtype=17), dict(dtype=-1), dict(idt=rd.RD_FP32),
               dict(first=-1), dict(scale=math.inf), dict(scale=math.nan), dict(out=P + 16), dict(out=4 * P), dict(tstride=1 << 60)):
        assert call(**kw) == bad, kw
    for kw in (dict(dtype=rd.RD_INT32), dict(dtype=rd.RD_FP64), dict(n=1 << 31), dict(rows=1 << 31)):
        assert call(**kw) == rd.RD_ERR_UNSUPPORTED, kw


def test_embed_grad_refusals():
    L, need = rd.lib(), C.c_size_t()
    assert L.rd_embed_grad_workspace(16, 8, 4, C.byref(need)) == rd.RD_OK and need.value > 0
    assert L.rd_embed_grad_workspace(16, 8, 4, None) == rd.RD_ERR_INVALID_ARG
    assert L.rd_embed_grad_workspace(0, 8, 4, C.byref(need)) == rd.RD_ERR_INVALID_ARG
    assert L.rd_embed_grad_workspace(1 << 32, 8, 4, C.byref(need)) == rd.RD_ERR_UNSUPPORTED

    def call(grad=P, gstride=8, dtype=rd.RD_BF16, ids=4 * P, idt=rd.RD_INT32, n=4, first=0, scale=1.0, table=2 * P, tstride=8, tdt=rd.RD_FP32, rows=16, dim=8, ws=8 * P,
             size=need.value):
        return L.rd_embed_grad(grad, gstride, dtype, ids, idt, n, first, scale, table, tstride, tdt, rows, dim, 0, ws, size, None)

    for kw in (dict(grad=None), dict(ids=None), dict(table=None), dict(ws=None), dict(ws=8 * P + 128), dict(grad=P + 1), dict(table=2 * P + 2), dict(ids=4 * P + 2),
               dict(gstride=7), dict(tstride=7), dict(tstride=0), dict(rows=0), dict(dim=0), dict(dtype=9), dict(tdt=9), dict(idt=rd.RD_BF16), dict(first=-1),
               dict(scale=math.inf), dict(table=P), dict(ws=P), dict(ws=4 * P), dict(ws=2 * P)):
        assert call(**kw) == rd.RD_ERR_INVALID_ARG, kw
    for kw in (dict(dtype=rd.RD_FP32, tdt=rd.RD_BF16), dict(dtype=rd.RD_BF16, tdt=rd.RD_FP16), dict(dtype=rd.RD_INT64, tdt=rd.RD_INT64), dict(n=1 << 31)):
        assert call(**kw) == rd.RD_ERR_UNSUPPORTED, kw
    assert call(size=need.value - 1) == rd.RD_ERR_TOO_SMALL


def vocab_struct(hidden=P, hs=8, weight=2 * P, ws=8, labels=4 * P, n=4, rows=16, dim=8, first=0, dtype=rd.RD_BF16, lt=rd.RD_INT64, scale=1.0, z=0.0):
    return rd.rd_vocab_t(hidden, hs, weight, ws, labels, n, rows, dim, first, dtype, lt, scale, z)


BAD_VOCAB = (dict(hidden=None), dict(weight=None), dict(labels=None), dict(hidden=P + 1), dict(weight=2 * P + 1), dict(labels=4 * P + 4), dict(hs=7), dict(ws=7), dict(ws=0),
             dict(rows=0), dict(dim=0), dict(dim=65537, hs=65537, ws=65537), dict(first=-1), dict(dtype=12), dict(lt=rd.RD_FP16), dict(scale=math.inf), dict(scale=0.0), dict(z=math.nan))


def test_vocab_loss_refusals():
    L, need = rd.lib(), C.c_size_t()
    assert L.rd_vocab_loss_workspace(C.byref(vocab_struct()), C.byref(need)) == rd.RD_OK and need.value > 0
    assert L.rd_vocab_loss_workspace(None, C.byref(need)) == rd.RD_ERR_INVALID_ARG
    assert L.rd_vocab_loss_workspace(C.byref(vocab_struct()), None) == rd.RD_ERR_INVALID_ARG

    def call(loss=16 * P, lse=17 * P, target=18 * P, ws=32 * P, size=need.value, **kw):
        return L.rd_vocab_loss(C.byref(vocab_struct(**kw)), loss, lse, target, ws, size, None)

    for kw in BAD_VOCAB + (dict(loss=None, lse=None, target=None), dict(loss=16 * P + 2), dict(ws=None), dict(ws=32 * P + 8), dict(loss=P), dict(lse=2 * P),
                           dict(target=4 * P), dict(lse=16 * P + 8), dict(ws=P), dict(ws=17 * P)):
        assert call(**kw) == rd.RD_ERR_INVALID_ARG, kw
    for kw in (dict(dtype=rd.RD_FP32), dict(dtype=rd.RD_INT32), dict(rows=1 << 31), dict(n=1 << 31)):
        assert call(**kw) == rd.RD_ERR_UNSUPPORTED, kw
    assert call(size=need.value - 1) == rd.RD_ERR_TOO_SMALL
    assert call(n=0, hidden=None, labels=None) == rd.RD_OK


def test_no_tokens_need_no_workspace():
    L, need = rd.lib(), C.c_size_t(1)
    none = vocab_struct(n=0, hidden=None, labels=None)
    assert L.rd_vocab_loss_workspace(C.byref(none), C.byref(need)) == rd.RD_OK and need.value == 0
    need.value = 1
    assert L.rd_vocab_loss_grad_workspace(C.byref(none), 1, 0, C.byref(need)) == rd.RD_OK and need.value == 0


def test_vocab_loss_grad_refusals():
    L, need = rd.lib(), C.c_size_t()
    assert L.rd_vocab_loss_grad_workspace(C.byref(vocab_struct()), 1, 1, C.byref(need)) == rd.RD_OK and need.value > 0

    def call(lse=16 * P, up=17 * P, ustride=1, gh=18 * P, ghs=8, gw=19 * P, gws=8, ws=32 * P, size=need.value, **kw):
        return L.rd_vocab_loss_grad(C.byref(vocab_struct(**kw)), lse, up, ustride, gh, ghs, gw, gws, ws, size, None)

    for kw in BAD_VOCAB + (dict(lse=None), dict(up=None), dict(gh=None, gw=None), dict(gh=18 * P + 1), dict(gw=19 * P + 1), dict(ghs=7), dict(gws=7), dict(ghs=0), dict(ws=None),
                           dict(ws=32 * P + 8), dict(gh=P), dict(gw=2 * P), dict(gw=18 * P), dict(gh=16 * P), dict(ws=19 * P), dict(ustride=1 << 60)):
        assert call(**kw) == rd.RD_ERR_INVALID_ARG, kw
    for kw in (dict(dtype=rd.RD_FP64), dict(rows=1 << 31), dict(n=1 << 31)):
        assert call(**kw) == rd.RD_ERR_UNSUPPORTED, kw
    assert call(size=need.value - 1) == rd.RD_ERR_TOO_SMALL
    assert call(n=0, hidden=None, labels=None, gw=None) == rd.RD_OK
    assert L.rd_vocab_status(None) == rd.RD_ERR_INVALID_ARG


@gpu
def test_binding_refusals():
    t, ids = torch.zeros(4, 8, device="cuda"), torch.zeros(3, dtype=torch.int64, device="cuda")
    for f in (lambda: rd.rd_embed(t.cpu(), ids), lambda: rd.rd_embed(t, ids.cpu()), lambda: rd.rd_embed(t.T, ids), lambda: rd.rd_embed(t[0], ids),
              lambda: rd.rd_embed(t, ids, torch.zeros(2, 8, device="cuda")), lambda: rd.rd_embed(t, ids, torch.zeros(3, 8, device="cuda").half()),
              lambda: rd.rd_embed_grad(t, ids, t.clone()), lambda: rd.rd_embed_grad(t[:3], ids, torch.zeros(4, 7, device="cuda")),
              lambda: rd.rd_vocab_loss(t[:3].half(), t, ids), lambda: rd.rd_vocab_loss(t.half(), t.half(), ids),
              lambda: rd.rd_vocab_loss_grad(t[:3].half(), t.half(), ids, ids.float(), ids.double(), None, t.half())):
        with pytest.raises(ValueError):
            f()
    for f in (lambda: rd.rd_vocab_loss(t[:3], t, ids), lambda: rd.rd_embed(t.double(), ids), lambda: rd.rd_embed_grad(t[:3].half(), ids, t.bfloat16())):
        with pytest.raises(rd.RdError) as e:
            f()
        assert e.value.status == rd.RD_ERR_UNSUPPORTED


# ------------------------------------------------------------------------------------------------ the operators together


@gpu
@pytest.mark.parametrize("processes, algo", [(1, rd.RD_UNI_GREEDY), (4, rd.RD_UNI_GREEDY), (3, rd.RD_BINOMIAL), (8, rd.RD_BI_GREEDY)])
def test_step_over_processes(processes, algo):
    """A step on a vocabulary cut over processes against the same step on the whole table in 64 bits."""
    from paper_1310_4645_b200.vocab_step import VocabStep
    rows, dim, n = 96 * processes, 48, 70
    table = rand(rows, dim, seed=120, dtype=torch.bfloat16, std=0.3)
    ids, labels = ints(0, rows, n, seed=121), ints(0, rows, n, seed=122)
    labels[::5] = -100
    step = VocabStep(table, processes, n, algo)
    try:
        loss, grads = step.run(ids, labels, embed_scale=3.0, logit_scale=0.5, z_loss=1e-3)
        w = table.double().requires_grad_()
        h = w[ids] * 3.0
        x = h @ w.T * 0.5
        lse = torch.logsumexp(x, 1)
        counts = labels >= 0
        t = x.gather(1, labels.clamp(min=0)[:, None])[:, 0]
        want = (torch.where(counts, lse - t + 1e-3 * lse * lse, 0.0)).sum() / counts.sum()
        want.backward()
        # the embedding is rounded to 16 bits once (only one process holds a row): x by 2^-8 of the magnitudes it sums, on average
        # over dim terms of either sign far less; the loss inherits that absolutely
        size = (h.abs() @ w.abs().T * 0.5).max().item()
        assert abs(loss.item() - want.item()) <= 2.0 ** -8 * size
        # gradients: five roundings to 16 bits (embedding, dx, dh per process, their sum, result), and probabilities off by 2^-8 * size
        got = torch.cat(grads).double()
        assert (got - w.grad).norm() <= (5 + size) * 2.0 ** -8 * w.grad.norm()
        assert rd.rd_vocab_status() == rd.RD_OK
    finally:
        step.close()


@gpu
def test_step_command(capsys):
    from paper_1310_4645_b200 import vocab_step
    vocab_step.main(["--processes", "2", "--vocab", "512", "--dim", "64", "--tokens", "100", "--steps", "4"])
    losses = [float(line.split()[3]) for line in capsys.readouterr().out.splitlines()]
    assert len(losses) == 4 and all(map(math.isfinite, losses)) and losses[-1] < losses[0]
