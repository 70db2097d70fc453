"""The vocabulary operators at the edges of their launches: shared memory, workspaces, paths that sizes alone decide, threads."""
import os
import shutil
import subprocess

import pytest
import torch

import paper_1310_4645_b200 as rd
from test_vocab import HALF, check_grad, check_loss, gen, vocab_case

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
