"""Calls of the block operators that their documentation allows or rules out, each on its own: activations, sums kept in 32 bits without a
residual, 8 bits into rows with a stride, shapes on the host."""
import pytest
import torch

import paper_1310_4645_b200 as rd
from test_vocab import rand

gpu = pytest.mark.gpu


@gpu
@pytest.mark.parametrize("activation", [-1, 3, 2 ** 31, 2 ** 32, 2 ** 32 + 2, -2 ** 32, 2 ** 62])
def test_activations_that_do_not_exist(activation):
    """Also those whose lower 32 bits name one."""
    x, w, d = (rand(*s, seed=1, dtype=torch.float16) for s in ((4, 8), (16, 8), (4, 16)))
    for call in (lambda: rd.rd_gated(x, w, w, activation), lambda: rd.rd_gated_grad(d, x, w, w, d, d, activation)):
        with pytest.raises(rd.RdError) as e:
            call()
        assert e.value.status == rd.RD_ERR_INVALID_ARG
