"""Calls of the block operators that their documentation allows or rules out, each on its own: activations, sums kept in 32 bits without a
residual, 8 bits into rows with a stride, shapes on the host."""
import os
import shutil
import subprocess

import pytest
import torch

import paper_1310_4645_b200 as rd
import test_norm
from test_norm import BF16, CSRC, E, E4M3, FP32, kept, norm_reference
from test_vocab import TINY, U, rand, within

gpu = pytest.mark.gpu

# every width of a tile and count of rows that the gated projections bring in, with and without the room where results change places
RINGS = r"""
#include <cstdio>
#include <initializer_list>
#include "rd_ring.h"
using namespace rd;
template <int CG> int check()
{
    int bad = 0;
    for (uint32_t a_rows = CG == 2 ? kRowsM : 8; a_rows <= kRowsM; a_rows += 8)
        for (uint32_t tile_w = 16; tile_w <= 128; tile_w += CG == 2 ? 16 : 8)
            for (const uint32_t staging : {0, kEpilogueWarps * 1024}) {
                const uint32_t room = Shape<kStats, CG>::ring - staging, columns = 2 * tile_w / CG;
                const Ring r = ring_of(room, a_rows, columns);
                // copies fill a stage; a product reads kRowsM rows of the left operand from its beginning, and the right one behind a_rows; swizzle
                // patterns begin on multiples of 1024 bytes
                const uint32_t last = (r.stages - 1) * r.stage, left = last + kRowsM * kTileK * 2, right = last + (a_rows + columns) * kTileK * 2;
                if (r.stages < 2 || r.stages > kMostStages || left > room || right > room || r.stage % 1024 || (a_rows * kTileK * 2) % 1024 || (tile_w * kTileK * 2) % 1024)
                    bad += std::printf("%d blocks: %u rows, %u columns, %u stages of %u\n", CG, a_rows, tile_w, r.stages, r.stage) > 0;
            }
    return bad;
}
int main() { return check<1>() + check<2>() != 0; }
"""


def run_on_the_host(tmp_path, source, *include):
    (tmp_path / "check.cpp").write_text(source)
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-I", CSRC, *include, "-o", str(tmp_path / "check"), str(tmp_path / "check.cpp")])
    done = subprocess.run([str(tmp_path / "check")], capture_output=True, text=True)
    assert done.returncode == 0, done.stdout[:2000]


def test_products_of_the_gated_projections_read_inside_the_ring(tmp_path):
    run_on_the_host(tmp_path, RINGS)


def test_rows_are_dealt_out_to_a_block_s_threads(tmp_path):
    """No deal has more threads than the kernels are built for, or more warps than have places in their shared arrays."""
    limit = "d.threads <= (unit_bytes ? 256 : 512)"
    assert limit in test_norm.DEALS
    include = os.path.join(os.path.dirname(shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"), "..", "include")
    run_on_the_host(tmp_path, test_norm.DEALS.replace(limit, "d.threads <= uint32_t(kThreads)"), "-I", include)


@gpu
@pytest.mark.parametrize("activation", [-1, 3, 2 ** 31, 2 ** 32, 2 ** 32 + 2, -2 ** 32, 2 ** 62])
def test_activations_that_do_not_exist(activation):
    """Also those whose lower 32 bits name one."""
    x, w, d = (rand(*s, seed=1, dtype=torch.float16) for s in ((4, 8), (16, 8), (4, 16)))
    for call in (lambda: rd.rd_gated(x, w, w, activation), lambda: rd.rd_gated_grad(d, x, w, w, d, d, activation)):
        with pytest.raises(rd.RdError) as e:
            call()
        assert e.value.status == rd.RD_ERR_INVALID_ARG


@gpu
@pytest.mark.parametrize("dim", [40, 256, 1000, 1001, 4096, 9000])
@pytest.mark.parametrize("drop", [0.0, 0.3])
def test_norm_keeps_its_sum_in_32_bits_without_a_residual(dim, drop):
    x, weight = rand(37, dim, seed=2, dtype=BF16), 1 + rand(1, dim, seed=3, std=0.3)[0]
    into = torch.full((37, dim), 7.0, device="cuda")
    out, total, rstd, _ = rd.rd_norm(x, weight, drop=drop, seed=4, total=into)
    s, err, r, rel = norm_reference(x, weight, None, 1e-6, kept(37, dim, drop, 4) if drop else 1.0)
    assert total is into
    within(total, s, err + U[FP32] * (s.abs() + err))
    within(rstd, r, rel * r)
    y = s * r[:, None] * weight.double()
    bound = y.abs() * (rel[:, None] + 3 * E) + err * (r[:, None] * weight.abs().double())
    within(out, y, bound + U[BF16] * (y.abs() + bound) + TINY[BF16])


@gpu
@pytest.mark.parametrize("dim", [24, 120, 1000, 1001, 4096, 9000])
@pytest.mark.parametrize("pad, offset", [(8, 0), (24, 8), (3, 1), (0, 5)])
def test_norm_into_8bit_rows_with_a_stride(dim, pad, offset):
    """The values where the rows say, nothing between and behind them."""
    n, weight = 21, 1 + rand(1, dim, seed=5, std=0.3)[0]
    x, residual = rand(n, dim, seed=6, dtype=BF16), rand(n, dim, seed=7)
    room = torch.full((n * (dim + pad) + offset + 16,), 0x55, dtype=torch.uint8, device="cuda")
    rows = room[offset:offset + n * (dim + pad)].view(n, dim + pad)[:, :dim]
    out, total, rstd, scale = rd.rd_norm(x, weight, residual, out_dtype=E4M3, out=rows.view(E4M3))
    s, err, r, rel = norm_reference(x, weight, residual, 1e-6, 1.0)
    y = s * r[:, None] * weight.double()
    most = y.abs().amax(1, keepdim=True)
    # the scale and the quotient inherit the row's relative errors (and the largest value's); then a rounding to half a step, 2^-10 below 2^-6
    e = (rel[:, None] + 8 * E) * 2 * y.abs() + 2 * err * r[:, None] * weight.abs().double()
    v, bv = y * (448 / most), e * (448 / most)
    within(out.float(), v, bv + 2.0 ** -4 * (v.abs() + bv) + 2.0 ** -10)
    within(scale, most[:, 0] / 448, e.amax(1) / 448 + 2.0 ** -149)
    rows.fill_(0x55)
    assert (room == 0x55).all()
