"""Rows of the norm that a cluster of thread blocks holds: more than 8192 columns, in the gradient of rows read by element more than 4096."""
import os
import re

import pytest
import torch

import paper_1310_4645_b200 as rd
import test_norm
from test_norm import BF16, CSRC, TYPES
from test_vocab import rand

gpu = pytest.mark.gpu


def test_blocks_of_a_cluster_have_begun_before_they_meet():
    """A block may write to another's shared memory only once that one has begun: every kernel whose rows may be a cluster's says that its
    blocks have begun, and waits for the others, before the first sum is joined.  (Read from the source: it cannot be tried out.)"""
    with open(os.path.join(CSRC, "rd_norm_kernels.h")) as f:
        source = re.sub(r"//.*", "", f.read())
    kernels = [k for k in re.split(r"__global__", source)[1:] if "join_row<WARP>" in k]
    assert len(kernels) == 2
    for k in kernels:
        begins, begun, meets = (k.find(name) for name in ("cluster_begins(p.blocks)", "cluster_has_begun(p.blocks)", "join_row<WARP>"))
        assert 0 <= begins < begun < meets
        # nobody leaves between the two, nor waits within the loop over rows
        assert "return" not in k[begins:begun] and begun < k.find("for (size_t row = at.row")


@gpu
@pytest.mark.parametrize("dtype, sum_dtype, weight_dtype", TYPES)
@pytest.mark.parametrize("n, dim, pad, offset", [(400, 8200, 0, 0), (400, 8193, 0, 0), (400, 16384, 0, 0), (400, 20001, 0, 0), (400, 5001, 3, 1), (130, 65536, 0, 0)])
def test_norm_grad_of_many_wide_rows(dtype, sum_dtype, weight_dtype, n, dim, pad, offset):
    """More rows than clusters fit at once, whose parts of the weight's gradient another launch joins."""
    test_norm.test_norm_grad(dtype, sum_dtype, weight_dtype, n, dim, pad, offset)


@gpu
@pytest.mark.parametrize("dim", [8200, 16384, 16381, 65536])
def test_clusters_beside_other_work(dim):
    """Calls of few rows while another stream keeps most of the SMs: the blocks of a cluster come up as room is made for them."""
    x, residual, weight, up = rand(3, dim, seed=1, dtype=BF16), rand(3, dim, seed=2, dtype=BF16), rand(1, dim, seed=3)[0], rand(3, dim, seed=4, dtype=BF16)

    def passes():
        out, total, rstd, _ = rd.rd_norm(x, weight, residual, drop=0.1, seed=5)
        return (out, total, rstd, *rd.rd_norm_grad(up, total, weight, rstd, residual, drop=0.1, seed=5))

    want = passes()
    other, a = torch.cuda.Stream(), rand(2048, 2048, seed=6, dtype=BF16)
    torch.cuda.synchronize()
    results = []
    with torch.cuda.stream(other):
        for _ in range(60):
            a @ a
    for _ in range(60):
        results.append(passes())
    torch.cuda.synchronize()
    assert all(torch.equal(g, w) for got in results for g, w in zip(got, want)) and rd.rd_block_status() == rd.RD_OK
