"""The vocabulary operators at the edges of their launches: shared memory, workspaces, paths that sizes alone decide, threads."""
import os
import shutil
import subprocess
import threading

import pytest
import torch

import paper_1310_4645_b200 as rd
import test_vocab
from test_vocab import HALF, U, check_grad, check_loss, gen, test_embed_grad_large_tables as large_tables, vocab_case, within

CSRC = os.path.join(os.path.dirname(os.path.abspath(rd.__file__)), "csrc")
gpu = pytest.mark.gpu

# every count of rows that a thread block brings in, every width of a tile, single blocks and pairs
RING = r"""
#include <cstdio>
#include "rd_ring.h"
using namespace rd;
template <int KIND, int CG> int check()
{
    int bad = 0;
    const uint32_t room = Shape<KIND, CG>::ring;
    for (uint32_t a_rows = CG == 2 ? kRowsM : 8; a_rows <= kRowsM; a_rows += 8)
        for (uint32_t columns = 64; columns <= kTileN; columns *= 2) {
            const Ring r = ring_of(room, a_rows, columns / CG);
            // copies fill a stage; a product reads kRowsM rows of the left operand from its beginning, and the right one behind a_rows
            const uint32_t last = (r.stages - 1) * r.stage, left = last + kRowsM * kTileK * 2, right = last + (a_rows + columns / CG) * kTileK * 2;
            if (r.stages < 2 || r.stages > kMostStages || right > r.stage * r.stages || right > room || left > room)
                bad += std::printf("kind %d, %d blocks: %u rows, %u columns: %u stages of %u, products read up to %u of %u\n", KIND, CG, a_rows, columns, r.stages, r.stage,
                                   left > right ? left : right, room) > 0;
        }
    return bad;
}
int main() { return check<kStats, 1>() + check<kStats, 2>() + check<kDlogits, 1>() + check<kDlogits, 2>() != 0; }
"""


def test_products_read_inside_the_ring(tmp_path):
    if not shutil.which("g++"):
        pytest.skip("no g++")
    (tmp_path / "ring.cpp").write_text(RING)
    subprocess.check_call(["g++", "-std=c++17", "-Wall", "-Werror", "-I", CSRC, "-o", str(tmp_path / "ring"), str(tmp_path / "ring.cpp")])
    r = subprocess.run([str(tmp_path / "ring")], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout


@gpu
@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("n", [25, 30, 32, 33])
def test_tokens_of_a_quarter_of_a_tile(dtype, n):
    """25 to 32 tokens, tiles of 64 columns and more steps than the ring has stages."""
    hidden, weight, labels = vocab_case(n, 9000, 1032, dtype, seed=200)
    check_loss(hidden, weight, labels)
    check_grad(hidden, weight, labels, torch.rand(n, generator=gen(201), device="cuda"))


def one_row(dim, stride, dtype=torch.bfloat16, device="cpu"):
    """A weight of one row, cut from a matrix whose rows are `stride` apart."""
    return torch.ones(3, stride, dtype=dtype, device=device)[:1, :dim]


@pytest.mark.parametrize("dim, stride", [(1000, 1001), (1001, 1008), (64, 64)])
def test_workspace_of_a_single_row(dim, stride):
    """What lies between rows is nothing to a matrix of one."""
    hidden, labels = torch.ones(3, dim, dtype=torch.bfloat16), torch.zeros(3, dtype=torch.int64)
    cut, alone = one_row(dim, stride), torch.ones(1, dim, dtype=torch.bfloat16)
    assert rd.rd_vocab_loss_workspace(hidden, cut, labels) == rd.rd_vocab_loss_workspace(hidden, alone, labels)
    assert rd.rd_vocab_loss_grad_workspace(hidden, cut, labels) == rd.rd_vocab_loss_grad_workspace(hidden, alone, labels)


@gpu
@pytest.mark.parametrize("dim, stride", [(1000, 1001), (1001, 1008)])
def test_workspace_of_a_single_row_suffices(dim, stride):
    weight = one_row(dim, stride, device="cuda")
    hidden, labels = torch.ones(3, dim, dtype=torch.bfloat16, device="cuda"), torch.zeros(3, dtype=torch.int64, device="cuda")
    ws = torch.empty(rd.rd_vocab_loss_workspace(hidden, weight, labels), dtype=torch.uint8, device="cuda")
    loss, lse, target = rd.rd_vocab_loss(hidden, weight, labels, workspace=ws)
    assert (target == dim).all()
    # the only logit times log2(e) and times ln(2) again: two constants and two products, each rounded to 2^-24
    assert (lse - dim).abs().max() <= dim * 2.0 ** -22 and loss.abs().max() <= dim * 2.0 ** -22
    ws = torch.empty(rd.rd_vocab_loss_grad_workspace(hidden, weight, labels), dtype=torch.uint8, device="cuda")
    up = torch.ones(3, device="cuda")
    gh, gw = rd.rd_vocab_loss_grad(hidden, weight, labels, lse, up, torch.empty_like(hidden), torch.empty_like(weight), workspace=ws)
    # the only entry has all of the probability: what is left is lse's error and that of the exponent, which is formed the same way
    assert gh.abs().max() <= dim * 2.0 ** -20 and gw.abs().max() <= 3 * dim * 2.0 ** -20


def lookup_overlaps(table, tstride, out, ostride, rows=16, n=4, dim=8, ids=1 << 24):
    """Whether rd_embed takes these addresses for overlapping memory.  They are no memory at all: without a device nothing is launched."""
    return rd.lib().rd_embed(table, tstride, rows, dim, rd.RD_BF16, ids, rd.RD_INT64, n, 0, 1.0, out, ostride, None) == rd.RD_ERR_INVALID_ARG


@pytest.mark.skipif(torch.cuda.is_available(), reason="calls with made-up addresses must find no device")
def test_columns_beside_each_other_do_not_overlap():
    P, row = 1 << 20, 48                                      # rows of 24 elements, in bytes
    assert not lookup_overlaps(P, 24, P + 16, 24)             # columns 0 to 7 and 8 to 15
    assert not lookup_overlaps(P + 32, 24, P, 24)             # 16 to 23 and 0 to 7
    assert not lookup_overlaps(P + 32, 24, P + row, 24)       # the same, from the next row on
    assert not lookup_overlaps(P, 24, P + 5 * row + 16, 24)
    assert not lookup_overlaps(P, 24, P + 5 * row + 16, 24, n=1) and not lookup_overlaps(P, 24, P + 5 * row + 16, 8, n=1)      # one row, whatever its stride
    assert lookup_overlaps(P, 24, P + 14, 24) and lookup_overlaps(P + 32, 24, P + 2, 24, dim=16)                              # columns that meet, in the next row too
    assert lookup_overlaps(P, 24, P + 5 * row + 14, 24, n=1) and lookup_overlaps(P, 24, P + 5 * row + 34, 24, n=1)            # 34: beyond the row's end
    assert lookup_overlaps(P, 24, P, 24) and lookup_overlaps(P, 24, P + 16, 32) and lookup_overlaps(P, 8, P + 16, 24)         # strides that differ
    assert lookup_overlaps(P, 24, P + 16, 24, ids=P + 16)     # the ids lie in the output


@gpu
def test_columns_of_one_buffer():
    """Operands and results side by side in one allocation."""
    n, rows, dim = 37, 61, 24
    buffer = torch.randn(rows, 5 * dim, device="cuda", generator=gen(210)).bfloat16()
    table, out, grad, grad_table, rest = (buffer[:, k * dim:(k + 1) * dim] for k in range(5))
    ids = torch.randint(0, rows, (n,), device="cuda", generator=gen(211))
    before = rest.clone()
    assert torch.equal(rd.rd_embed(table, ids, out[:n]), table.contiguous()[ids])
    want = rd.rd_embed_grad(grad[:n].contiguous(), ids, torch.empty(rows, dim, dtype=torch.bfloat16, device="cuda"))
    assert torch.equal(rd.rd_embed_grad(grad[:n], ids, grad_table), want)
    hidden, weight = grad[:n], table
    _, lse, _ = rd.rd_vocab_loss(hidden, weight, ids)
    up = torch.ones(n, device="cuda")
    fresh = rd.rd_vocab_loss_grad(hidden, weight, ids, lse, up, torch.empty(n, dim, dtype=torch.bfloat16, device="cuda"), torch.empty(rows, dim, dtype=torch.bfloat16, device="cuda"))
    got = rd.rd_vocab_loss_grad(hidden, weight, ids, lse, up, out[:n], grad_table)
    assert torch.equal(got[0], fresh[0]) and torch.equal(got[1], fresh[1]) and torch.equal(rest, before)


@gpu
@pytest.mark.parametrize("dtype, out, n, rows, dim, pad", [
    # sort on the library's stream, the whole table filled meanwhile, sums on the caller's stream after both:
    (torch.bfloat16, torch.bfloat16, 9001, 100003, 264, 0),       # 53 MB, rows through shared memory
    (torch.bfloat16, torch.float32, 30000, 30011, 512, 8),        # 61 MB and gaps between the rows
    (torch.bfloat16, torch.bfloat16, 6000, 450001, 40, 0),        # 36 MB, rows below 512 bytes
    (torch.float16, torch.float16, 6000, 60013, 333, 3),          # 40 MB, element by element
    (torch.float32, torch.float32, 5000, 700001, 100, 0),         # 280 MB, more than is filled first, but rows below 512 bytes
    # no fork: just below 32 MiB
    (torch.bfloat16, torch.bfloat16, 9001, 63000, 264, 0),
])
def test_table_gradient_filled_at_once(dtype, out, n, rows, dim, pad):
    large_tables(dtype, out, n, rows, dim, pad)


def within_type(got, want, bound):
    """within, for a result type whose largest finite number the definition's value may exceed."""
    most = torch.finfo(got.dtype).max
    over, under = want.abs() - bound > most * (1 + U[got.dtype]), want.abs() + bound < most
    assert torch.equal(got[over].double(), torch.copysign(torch.full_like(want, float("inf")), want)[over])
    within(got[under], want[under], bound[under])
    either = got[~over & ~under]
    assert (torch.isinf(either) | (either.double().abs() >= (want.abs() - bound)[~over & ~under])).all()


@gpu
@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("n", [1024, 1025, 4096, 4097, 5003])
def test_packed_tokens(dtype, n):
    """Blocks that pack one token (up to 1024) or eight, that count for themselves (up to 4096) or look at the tiles' counts; a dim that
    needs the weight's copy, and one that fills no step."""
    for rows, dim in ((701, 101), (300, 200)):
        hidden, weight, labels = vocab_case(n, rows, dim, dtype, seed=220)
        labels[-1] = rows - 1
        check_loss(hidden, weight, labels, scale=0.7, z=1e-2)
        up = (0.5 + torch.rand(n, generator=gen(221), device="cuda")) / n
        check_grad(hidden, weight, labels, up, z=1e-2)


@gpu
@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("n", [200, 1500, 5003])
@pytest.mark.parametrize("size", [1e-9, 1.0, 1e3])
def test_packed_sizes_of_the_upstream_gradient(dtype, n, size, monkeypatch):
    """The largest one in the last tile of tokens, or an ignored token's: fp16's power of two goes by the tokens that count."""
    # 64000 times a hidden value is beyond fp16: an infinity of its sign there, as one rounding of the definition's value gives
    monkeypatch.setattr(test_vocab, "within", within_type)
    hidden, weight, labels = vocab_case(n, 400, 72, dtype, seed=230)
    up = torch.rand(n, generator=gen(231), device="cuda") * size
    labels[-1], up[-1] = 7, 64 * size
    check_grad(hidden, weight, labels, up)
    labels[n // 2], up[n // 2] = -100, 2.0 ** 40
    up[-1] = size
    check_grad(hidden, weight, labels, up)


@gpu
def test_calls_from_threads():
    """Threads with streams of their own: two that want the library's second stream at once, one on the loss, one on small tables."""
    n, rows, dim = 9000, 40000, 512
    ids = torch.randint(0, rows, (n,), generator=gen(240), device="cuda")
    grads = [torch.randn(n, dim, generator=gen(241 + k), device="cuda").bfloat16() for k in range(2)]
    hidden, weight, labels = vocab_case(300, 2000, 64, torch.bfloat16, seed=243)
    up = torch.ones(300, device="cuda")

    def large(k):
        return lambda: (rd.rd_embed_grad(grads[k], ids, torch.full((rows, dim), 7.0, dtype=torch.bfloat16, device="cuda")),)

    def loss():
        out = rd.rd_vocab_loss(hidden, weight, labels)
        return (*out, *rd.rd_vocab_loss_grad(hidden, weight, labels, out[1], up, torch.empty_like(hidden), torch.empty_like(weight)))

    def small():
        return (rd.rd_embed(weight, labels), rd.rd_embed_grad(hidden, labels, torch.empty_like(weight)))

    calls = (large(0), large(1), loss, small)
    want = [f() for f in calls]
    torch.cuda.synchronize()
    ready, wrong = threading.Barrier(len(calls)), []

    def work(f, expected):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                ready.wait(60)
                got = [f() for _ in range(20)]
                torch.cuda.current_stream().synchronize()
            if not all(torch.equal(a, b) for out in got for a, b in zip(out, expected)):
                wrong.append("results differ")
        except Exception as e:
            wrong.append(repr(e))

    threads = [threading.Thread(target=work, args=c) for c in zip(calls, want)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong and rd.rd_vocab_status() == rd.RD_OK
