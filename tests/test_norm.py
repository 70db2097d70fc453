"""Root-mean-square norm with the residual's addition and dropout, its gradient, and dropout alone, against their definitions in 64 bits.

Bounds.  u is the unit round-off of the result's type (bf16 2^-8, fp16 2^-11, fp32 2^-24, e4m3 2^-4).  e = 2^-24 is a fp32 operation's.
s takes two operations (the factor of dropout, the residual's addition).  A row's sum adds up at most 32 values in a thread and then
pairs, warps and thread blocks: fewer than 64 additions on any value's way, each off by e of what has been added up.  rsqrt is within
2 units in the last place.
"""
import ctypes as C
import math
import os
import shutil
import subprocess

import numpy as np
import pytest
import torch

import paper_1310_4645_b200 as rd
from test_vocab import TINY, U, gen, ints, rand, strided, within

gpu = pytest.mark.gpu
CSRC = os.path.join(os.path.dirname(os.path.abspath(rd.__file__)), "csrc")
E = 2.0 ** -24
BF16, FP16, FP32, E4M3 = torch.bfloat16, torch.float16, torch.float32, torch.float8_e4m3fn
# rows' type, type of residual and sum, type of the weight
TYPES = [(BF16, BF16, BF16), (BF16, FP32, FP32), (FP16, FP16, FP32), (FP16, FP32, FP16), (FP32, FP32, FP32)]


def philox(counter, key):
    """Philox 4x32 with 10 rounds on arrays of four counter words and two key words."""
    a, b, c, d = (np.asarray(w, dtype=np.uint64) for w in counter)
    k0, k1 = (np.asarray(w, dtype=np.uint64) for w in key)
    low = np.uint64(0xFFFFFFFF)
    for _ in range(10):
        x, y = a * np.uint64(0xD2511F53), c * np.uint64(0xCD9E8D57)
        a, b, c, d = (y >> np.uint64(32)) ^ b ^ k0, y & low, (x >> np.uint64(32)) ^ d ^ k1, x & low
        k0, k1 = (k0 + np.uint64(0x9E3779B9)) & low, (k1 + np.uint64(0xBB67AE85)) & low
    return a, b, c, d


def test_generator_of_the_tests():
    """Published answers of the generator."""
    hexes = lambda words: " ".join("%08x" % int(w) for w in words)
    assert hexes(philox([0] * 4, [0] * 2)) == "6627e8d5 e169c58d bc57ac4c 9b00dbd8"
    assert hexes(philox([0xFFFFFFFF] * 4, [0xFFFFFFFF] * 2)) == "408f276d 41c83b0e a20bc7c6 6d5451fd"
    assert hexes(philox([0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344], [0xA4093822, 0x299F31D0])) == "d16cfe09 94fdcceb 5001e420 24126ea1"


def kept(n, dim, drop, seed=0, offset=0, first=0):
    """What dropout multiplies by, [n, dim] in 64 bits."""
    border = round(float(np.float32(drop)) * 65536)
    units = (dim + 7) // 8
    i, j = np.meshgrid(np.arange(n, dtype=np.uint64) + np.uint64(first), np.arange(units, dtype=np.uint64), indexing="ij")
    low = 0xFFFFFFFF
    words = philox([j, i, np.full_like(i, offset & low), np.full_like(i, offset >> 32)], [np.full_like(i, seed & low), np.full_like(i, seed >> 32)])
    bits = np.stack([w >> np.uint64(s) & np.uint64(0xFFFF) for w in words for s in (0, 16)], -1).reshape(n, units * 8)[:, :dim]
    factor = float(np.float32(65536 / (65536 - border)))
    return torch.from_numpy((bits >= border) * factor).cuda()


DEALS = r"""
#include <cstdio>
#include "rd_norm_shape.h"
using namespace rd;
int main()
{
    int bad = 0;
    for (size_t dim = 1; dim <= 65536; dim++)
        for (const size_t unit_bytes : {0, 16, 32, 48, 64, 80, 96})
            for (const bool few : {false, true}) {
                const RowDeal d = deal(dim, unit_bytes, few);
                const RowShape s = shape_of(1000, d, unit_bytes);
                const size_t all = size_t(d.per_block) * d.blocks, threads = d.lanes ? d.lanes : d.warp ? 32 : d.threads;
                // every unit is somebody's, every block has some, no thread more than its registers hold, no stage beyond the ring
                bool ok = all >= d.units && all - d.per_block < d.units && size_t(d.nv) * threads >= d.per_block && d.blocks <= 8 && (d.blocks == 1 || d.per_block % 32 == 0);
                ok = ok && d.threads % 32 == 0 && d.threads <= (unit_bytes ? 256 : 512) && (d.warp || d.threads >= 64) && s.groups > 0;
                if (unit_bytes && !d.lanes) ok = ok && s.ring.stages >= 2 && s.ring.stages <= kMostStages && s.ring.stage >= d.per_block * unit_bytes && s.smem <= kRingBytes && s.smem >= size_t(s.ring.stages) * s.ring.stage * (d.warp ? kWarps : 1);
                if (!ok) bad += std::printf("dim %zu, %zu bytes, few %d\n", dim, unit_bytes, few) > 0;
            }
    return bad != 0;
}
"""


def test_rows_are_dealt_out(tmp_path):
    """Which threads have which columns, and the shared memory that rows come in through, for every row length, on the host."""
    source, program = tmp_path / "deals.cpp", tmp_path / "deals"
    source.write_text(DEALS)
    include = ["-I", CSRC, "-I", os.path.join(os.path.dirname(shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"), "..", "include")]
    subprocess.check_call(["g++", "-std=c++17", "-O1", *include, "-o", str(program), str(source)])
    done = subprocess.run([str(program)], capture_output=True, text=True)
    assert done.returncode == 0, done.stdout[:2000]


# ------------------------------------------------------------------------------------------------ dropout


@gpu
@pytest.mark.parametrize("dtype", [BF16, FP16, FP32])
@pytest.mark.parametrize("n, dim, pad, offset", [(1, 1, 0, 0), (1, 8, 0, 0), (3, 7, 0, 0), (5, 64, 0, 0), (33, 65, 0, 0), (300, 1000, 0, 0), (70, 1000, 8, 0), (70, 1000, 3, 1),
                                                 (2, 8200, 0, 0), (3, 8193, 0, 0), (1, 65536, 0, 0), (70000, 8, 0, 0), (66000, 5, 0, 0)])
def test_dropout(dtype, n, dim, pad, offset):
    x = strided(rand(n, dim, seed=1, dtype=dtype), pad, offset)
    for drop, seed, shift, first in ((0.3, 2 ** 64 - 3, 2 ** 40 + 7, 5), (0.5, 1, 0, 2 ** 32 - n), (2.0 ** -16, 12345678901, 2 ** 64 - 1, 0)):
        want = x.double() * kept(n, dim, drop, seed, shift, first)
        out = strided(torch.full((n, dim), 7.0, dtype=dtype, device="cuda"), pad, offset)
        assert rd.rd_dropout(x, drop, seed, shift, first_row=first, out=out) is out
        within(out, want, (U[dtype] + E) * want.abs() + TINY[dtype])
        assert torch.equal(out == 0, (want == 0) | (x == 0))
        assert torch.equal(rd.rd_dropout(x, drop, seed, shift, first_row=first), out)
        # in place
        again = strided(x, pad, offset)
        assert rd.rd_dropout(again, drop, seed, shift, first_row=first, out=again) is again and torch.equal(again, out)
    assert torch.equal(rd.rd_dropout(x, 0.0, 3), x)


@gpu
def test_dropout_slices():
    """Rows of a slice draw what they draw in the whole; other seeds, offsets and rows draw something else."""
    x = torch.ones(64, 256, device="cuda")
    whole = rd.rd_dropout(x, 0.5, 9, 4)
    assert torch.equal(torch.cat([rd.rd_dropout(x[a:b], 0.5, 9, 4, first_row=a) for a, b in ((0, 1), (1, 40), (40, 64))]), whole)
    for other in (rd.rd_dropout(x, 0.5, 10, 4), rd.rd_dropout(x, 0.5, 9, 5), rd.rd_dropout(x, 0.5, 9, 4, first_row=64), rd.rd_dropout(x, 0.5, 9 + 2 ** 32, 4),
                  rd.rd_dropout(x, 0.5, 9, 4 + 2 ** 32)):
        # 16384 fair coins agree 8192 times, give or take 64 = one standard deviation
        assert abs((other == whole).sum().item() - 8192) < 8 * 64
    for drop in (0.1, 0.9):
        share = (rd.rd_dropout(x, drop, 11) == 0).float().mean().item()
        assert abs(share - drop) < 8 * math.sqrt(0.09 / 16384)
    # a broadcast row, infinities and NaN in dropped places
    one = torch.full((1, 256), math.nan, device="cuda").expand(64, 256)
    out = rd.rd_dropout(one, 0.5, 9, 4)
    assert torch.equal(torch.isnan(out), whole != 0) and not out[whole == 0].any()


# ------------------------------------------------------------------------------------------------ norm


def norm_reference(x, weight, residual, eps, keep):
    """(s, bound of s, rstd, relative bound of rstd) in 64 bits."""
    s = x.double() * keep
    err = E * s.abs()
    if residual is not None:
        s = s + residual.double()
        err = err + E * s.abs()
    square = s.square().mean(1) + eps
    rel = (2 * (s.abs() * err).mean(1) + 70 * E * s.square().mean(1)) / square + 3 * E
    return s, err, square.rsqrt(), rel / 2 + 2.0 ** -22


NORM_SHAPES = [(1, 1, 0, 0), (1, 8, 0, 0), (3, 7, 0, 0), (9, 64, 0, 0), (20, 65, 0, 0), (8, 256, 0, 0), (9, 264, 8, 0), (17, 512, 0, 0), (40, 1000, 0, 0), (40, 1000, 3, 1), (31, 1024, 0, 0),
               (33, 1025, 0, 0), (33, 1032, 0, 0), (5, 2048, 0, 0), (5, 2056, 8, 8), (300, 4096, 0, 0), (3, 8192, 0, 0), (3, 8200, 0, 0), (3, 8193, 0, 0), (2, 16384, 0, 0),
               (2, 20001, 0, 0), (3, 65536, 0, 0), (2, 65535, 0, 0), (5000, 72, 0, 0),
               (700, 8, 0, 0), (33, 48, 8, 8), (5, 128, 0, 0), (700, 120, 8, 0), (129, 136, 0, 0), (2, 3048, 0, 0), (2, 8240, 0, 0), (2, 12320, 0, 0), (3, 24584, 0, 0)]


@gpu
@pytest.mark.parametrize("dtype, sum_dtype, weight_dtype", TYPES)
@pytest.mark.parametrize("n, dim, pad, offset", NORM_SHAPES)
def test_norm(dtype, sum_dtype, weight_dtype, n, dim, pad, offset):
    x = strided(rand(n, dim, seed=2, dtype=dtype), pad, offset)
    weight = (1 + rand(1, dim, seed=3, std=0.3)[0]).to(weight_dtype)
    residual = strided(rand(n, dim, seed=4, dtype=sum_dtype, std=3.0), pad, offset)
    w = weight.double()
    for res, drop in ((None, 0.0), (residual, 0.0), (residual, 0.2), (None, 0.4)):
        if res is None and sum_dtype != dtype:
            continue
        keep = kept(n, dim, drop, 77, 88, 99) if drop else 1.0
        s, err, rstd, rel = norm_reference(x, weight, res, 1e-5, keep)
        out = strided(torch.full((n, dim), 7.0, dtype=dtype, device="cuda"), pad, offset)
        args = dict(eps=1e-5, drop=drop, seed=77, offset=88, first_row=99)
        got, total, r, scale = rd.rd_norm(x, weight, res, out=out, **args)
        assert got is out and scale is None and (total is None) == (res is None and not drop)
        if total is not None:
            within(total, s, err + U[sum_dtype] * (s.abs() + err) + TINY[sum_dtype])
        within(r, rstd, rel * rstd)
        y = s * rstd[:, None] * w
        bound = y.abs() * (rel[:, None] + 3 * E) + err * (rstd[:, None] * w.abs())
        within(out, y, bound + U[dtype] * (y.abs() + bound) + TINY[dtype])
        # eight bits: the scale inherits the relative bounds of its row, the quotient is rounded to half a step, 2^-10 below 2^-6
        q, total8, r8, scale = rd.rd_norm(x, weight, res, out_dtype=E4M3, **args)
        assert q.dtype == E4M3 and torch.equal(r8, r) and (total is None or torch.equal(total8, total))
        most = y.abs().amax(1)
        bm = bound.amax(1) + 3 * E * most
        within(scale, most / 448, bm / 448 + 2.0 ** -149)
        v = y * (448 / most.clamp(min=1e-300))[:, None]
        bv = 448 * (bound / most.clamp(min=1e-300)[:, None]) + v.abs() * (bm / most.clamp(min=1e-300))[:, None] + 4 * E * v.abs()
        within(q.float(), v, bv + 2.0 ** -4 * (v.abs() + bv) + 2.0 ** -10)


@gpu
@pytest.mark.parametrize("dim", [40, 128, 256, 1024, 1041, 4096, 9000])
def test_norm_in_place(dim):
    """out may be x, the sum may be the residual or x; the bits do not change."""
    x, residual, weight = rand(19, dim, seed=5, dtype=BF16), rand(19, dim, seed=6, dtype=BF16), rand(1, dim, seed=7, dtype=BF16)[0]
    out, total, rstd, _ = rd.rd_norm(x, weight, residual, drop=0.1, seed=3)
    for into, sum_into in ((None, "residual"), ("x", "residual"), (None, "x"), ("residual", "x")):
        t = {"x": x.clone(), "residual": residual.clone()}
        o, s, r, _ = rd.rd_norm(t["x"], weight, t["residual"], drop=0.1, seed=3, out=t.get(into), total=t[sum_into])
        assert s is t[sum_into] and torch.equal(o, out) and torch.equal(s, total) and torch.equal(r, rstd)
    wide = residual.float()
    o, s, _, _ = rd.rd_norm(x, weight, wide.clone())
    t = wide.clone()
    o2, s2, _, _ = rd.rd_norm(x, weight, t, total=t)
    assert s2 is t and torch.equal(o, o2) and torch.equal(s, s2)


@gpu
@pytest.mark.parametrize("dim", [64, 120, 256, 2000, 2001])
def test_norm_special_rows(dim):
    """Rows of zeros, infinities, NaN, very large and very small values, each on its own."""
    x = rand(8, dim, seed=8)
    x[1] = 0
    x[2, 5] = math.inf
    x[3, 6] = math.nan
    x[4] *= 1e-18
    x[5] *= 1e16
    x[6] = 0
    x[6, 3] = -2.0
    weight = torch.ones(dim, device="cuda")
    out, total, rstd, _ = rd.rd_norm(x, weight, eps=1e-6)
    assert total is None and not out[1].any() and abs(rstd[1].item() - 1000) < 1e-3
    assert rstd[2] == 0 and torch.isnan(out[2, 5]) and not out[2, torch.arange(dim, device="cuda") != 5].any()
    assert torch.isnan(rstd[3]) and torch.isnan(out[3]).all()
    assert torch.isfinite(out[[0, 1, 4, 5, 6, 7]]).all()
    unit = out[5].double().square().mean().item()
    assert abs(unit - 1) < 1e-5
    q, _, _, scale = rd.rd_norm(x, weight, eps=1e-6, out_dtype=E4M3)
    assert scale[1] == 0 and not q[1].float().any()
    assert torch.isnan(scale[[2, 3]]).all() and torch.isfinite(scale[[0, 1, 4, 5, 6, 7]]).all()
    assert q[6, 3].float() == -448 and q[6].float().abs().sum() == 448
    for row in (0, 4, 5, 7):
        assert q[row].float().abs().max() == 448
        value = q[row].double() * scale[row].double()
        assert (value - out[row].double()).abs().max() <= (2.0 ** -4 + 1e-5) * out[row].abs().max().item()
    # without eps a row of zeros is 0 / 0
    out, _, rstd, _ = rd.rd_norm(x, weight, eps=0.0)
    assert torch.isinf(rstd[1]) and torch.isnan(out[1]).all() and torch.isfinite(out[0]).all()
    # values so small that their squares vanish: eps alone decides
    tiny = torch.full((1, dim), 1e-30, device="cuda")
    out, _, _, _ = rd.rd_norm(tiny, weight, eps=1e-6)
    assert torch.allclose(out, tiny * 1000, rtol=1e-6, atol=0)
    q, _, _, scale = rd.rd_norm(tiny, weight, eps=1e-6, out_dtype=E4M3)
    assert (q.float() == 448).all() and abs(scale.item() * 448e27 - 1) < 1e-5


# ------------------------------------------------------------------------------------------------ gradient of the norm


@gpu
@pytest.mark.parametrize("dtype, sum_dtype, weight_dtype", TYPES)
@pytest.mark.parametrize("n, dim, pad, offset", NORM_SHAPES + [(1000, 1024, 0, 0), (600, 1200, 0, 0), (700, 333, 0, 0), (384, 264, 0, 0), (385, 265, 0, 0), (384, 2000, 3, 1), (385, 2000, 8, 0)])
def test_norm_grad(dtype, sum_dtype, weight_dtype, n, dim, pad, offset):
    up = strided(rand(n, dim, seed=11, dtype=dtype), pad, offset)
    total = strided(rand(n, dim, seed=12, dtype=sum_dtype, std=2.0), pad, offset)
    weight = (1 + rand(1, dim, seed=13, std=0.3)[0]).to(weight_dtype)
    more = strided(rand(n, dim, seed=14, dtype=sum_dtype), pad, offset)
    rstd = (total.double().square().mean(1) + 1e-5).rsqrt().float()
    r, s, u, w = rstd.double()[:, None], total.double(), up.double(), weight.double()
    normed, g = s * r, u * w
    mean = (g * normed).mean(1, keepdim=True)
    base = r * (g - normed * mean)
    # the mean: two products and fewer than 70 additions; then the difference, a product and the sum
    bm = (g * normed).abs().mean(1, keepdim=True) * 75 * E
    bb = r * (g.abs() * 3 * E + normed.abs() * (bm + mean.abs() * 4 * E)) + 2 * E * base.abs()
    for extra, drop in ((None, 0.0), (more, 0.0), (more, 0.3)):
        grad = base if extra is None else base + extra.double()
        bg = bb + E * grad.abs()
        keep = kept(n, dim, drop, 5, 6, 7) if drop else 1.0
        gx = strided(torch.full((n, dim), 7.0, dtype=dtype, device="cuda"), pad, offset)
        gr = strided(torch.full((n, dim), 7.0, dtype=sum_dtype, device="cuda"), pad, offset)
        args = dict(drop=drop, seed=5, offset=6, first_row=7)
        a, b, gw = rd.rd_norm_grad(up, total, weight, rstd, extra, grad_x=gx, grad_residual=gr, **args)
        assert a is gx and b is gr
        within(gr, grad, bg + U[sum_dtype] * (grad.abs() + bg) + TINY[sum_dtype])
        want = grad * keep
        bx = bg * keep + E * want.abs()
        within(gx, want, bx + U[dtype] * (want.abs() + bx) + TINY[dtype])
        total_w = (u * normed).sum(0)
        bw = (u * normed).abs().sum(0) * (min(n, 600) + 80) * E
        within(gw, total_w, bw + U[weight_dtype] * (total_w.abs() + bw) + TINY[weight_dtype])
        # one at a time, the same bits
        x1, r1, w1 = rd.rd_norm_grad(up, total, weight, rstd, extra, want_residual=False, want_weight=False, **args)
        assert r1 is None and w1 is None and torch.equal(x1, gx)
        x2, r2, w2 = rd.rd_norm_grad(up, total, weight, rstd, extra, **args)
        assert torch.equal(w2, gw) and torch.equal(r2, gr) and torch.equal(x2, gx) and (r2 is x2) == (not drop and dtype == sum_dtype)


@gpu
@pytest.mark.parametrize("n", [50, 500])
def test_norm_grad_weight_alone_and_no_rows(n):
    L = rd.lib()
    up, total, weight = rand(n, 96, seed=15), rand(n, 96, seed=16), rand(1, 96, seed=17)[0]
    rstd = torch.ones(n, device="cuda")
    _, _, want = rd.rd_norm_grad(up, total, weight, rstd)
    got = torch.empty_like(weight)
    ws = torch.empty(rd.rd_norm_grad_workspace(n, 96), dtype=torch.uint8, device="cuda")
    v = rd.rd_norm_grad_t(up.data_ptr(), 96, total.data_ptr(), 96, rstd.data_ptr(), weight.data_ptr(), None, 0, n, 96, rd.RD_FP32, rd.RD_FP32, rd.RD_FP32, 0.0, 0, 0, 0)
    stream = torch.cuda.current_stream().cuda_stream
    assert L.rd_norm_grad(C.byref(v), None, 0, None, 0, got.data_ptr(), ws.data_ptr() if ws.numel() else None, ws.numel(), stream) == rd.RD_OK
    assert torch.equal(got, want)
    x, r, w = rd.rd_norm_grad(up[:0], total[:0], weight, rstd[:0])
    assert x.shape == (0, 96) and not w.any()
    out, total, rstd, scale = rd.rd_norm(up[:0], weight, up[:0], out_dtype=E4M3)
    assert out.shape == total.shape == (0, 96) and rstd.shape == scale.shape == (0,)
    assert rd.rd_dropout(up[:0], 0.5, 1).shape == (0, 96)


@gpu
@pytest.mark.parametrize("n", [21, 384, 385])
@pytest.mark.parametrize("dim", [24, 128, 1040, 1041, 8208])
def test_norm_grad_in_place(n, dim):
    up, total, more = (rand(n, dim, seed=18 + k, dtype=BF16) for k in range(3))
    weight, rstd = rand(1, dim, seed=21, dtype=BF16)[0], torch.rand(n, generator=gen(22), device="cuda")
    gx, gr, gw = rd.rd_norm_grad(up, total, weight, rstd, more, drop=0.2, seed=1)
    for x_into, r_into in ((0, 1), (1, 2), (2, 0), (0, 2)):
        t = [up.clone(), total.clone(), more.clone()]
        a, b, w = rd.rd_norm_grad(t[0], t[1], weight, rstd, t[2], drop=0.2, seed=1, grad_x=t[x_into], grad_residual=t[r_into])
        assert a is t[x_into] and b is t[r_into] and torch.equal(a, gx) and torch.equal(b, gr) and torch.equal(w, gw)


@gpu
def test_norm_grad_is_the_derivative():
    """Difference quotients of <a, out> + <b, total> under dropout with respect to x, the residual and the weight."""
    n, dim, eps, h = 4, 24, 1e-3, 2.0 ** -6
    x, residual, a, b = (rand(n, dim, seed=30 + k) for k in range(4))
    weight = 1 + rand(1, dim, seed=34, std=0.3)[0]
    args = dict(drop=0.25, seed=42, offset=1, first_row=3)

    def value(x, residual, weight):
        out, total, _, _ = rd.rd_norm(x, weight, residual, eps=eps, **args)
        return (out.double() * a.double() + total.double() * b.double()).sum().item()

    out, total, rstd, _ = rd.rd_norm(x, weight, residual, eps=eps, **args)
    gx, gr, gw = rd.rd_norm_grad(a, total, weight, rstd, b, **args)
    size = (a.abs().double() * out.abs().double() + b.abs().double() * total.abs().double()).sum().item()
    # rounding: about ten operations a value, over 2 h; the third derivative is at most some 10 (rows of length about sqrt(dim), a and
    # weights of a few), times h^2 / 6
    bound = 10 * E * size / h + 10 * 10 * h * h / 6
    for i, j in ((0, 0), (1, 7), (3, 23), (2, 11)):
        for k, g in ((0, gx), (1, gr)):
            moved = [[x.clone(), residual.clone()] for _ in range(2)]
            moved[0][k][i, j] += h
            moved[1][k][i, j] -= h
            quotient = (value(*moved[0], weight) - value(*moved[1], weight)) / (2 * h)
            assert abs(quotient - g[i, j].item()) <= bound
        moved = [weight.clone(), weight.clone()]
        moved[0][j] += h
        moved[1][j] -= h
        assert abs((value(x, residual, moved[0]) - value(x, residual, moved[1])) / (2 * h) - gw[j].item()) <= bound


@gpu
@pytest.mark.parametrize("dim", [128, 4096, 10000])
def test_norm_streams_and_graphs(dim):
    """On a stream of its own, and recorded and played again on other inputs, with the bits of the plain calls."""
    x, residual, weight, up = rand(37, dim, seed=50, dtype=BF16), rand(37, dim, seed=51, dtype=BF16), rand(1, dim, seed=52, dtype=BF16)[0], rand(37, dim, seed=53, dtype=BF16)
    args = dict(drop=0.1, seed=7, offset=8)

    def passes(stream=None):
        out, total, rstd, _ = rd.rd_norm(x, weight, residual, stream=stream, **args)
        return (out, total, rstd, *rd.rd_norm_grad(up, total, weight, rstd, residual, stream=stream, **args), rd.rd_dropout(x, 0.1, 7, stream=stream))

    want = passes()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = passes(side)
    torch.cuda.synchronize()
    assert all(map(torch.equal, got, want))
    kept_x = x.clone()
    x.zero_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = passes()
    x.copy_(kept_x)
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    assert all(map(torch.equal, got, want))


# ------------------------------------------------------------------------------------------------ refusals


P = 1 << 20                                                   # made-up addresses: everything below is refused before a launch


def refused(call, good, bad, unsupported):
    for kw in bad:
        assert call(**{**good, **kw}) == rd.RD_ERR_INVALID_ARG, kw
    for kw in unsupported:
        assert call(**{**good, **kw}) == rd.RD_ERR_UNSUPPORTED, kw


def test_norm_refusals():
    L = rd.lib()

    def call(out, out_stride, out_type, scale, sum, sum_stride, rstd, **kw):
        return L.rd_norm(C.byref(rd.rd_norm_t(*kw.values())), out, out_stride, out_type, scale, sum, sum_stride, rstd, None)

    good = dict(out=3 * P, out_stride=8, out_type=rd.RD_BF16, scale=None, sum=4 * P, sum_stride=8, rstd=5 * P, x=P, xs=8, residual=2 * P, rs=8, weight=6 * P, n=4, dim=8,
                dtype=rd.RD_BF16, sum_dtype=rd.RD_BF16, weight_dtype=rd.RD_BF16, eps=1e-6, drop=0.0, seed=0, offset=0, first=0)
    refused(call, good, [dict(x=None), dict(weight=None), dict(out=None), dict(x=P + 1), dict(weight=6 * P + 1), dict(residual=2 * P + 1), dict(out=3 * P + 1), dict(sum=4 * P + 1),
                         dict(rstd=5 * P + 2), dict(xs=7), dict(rs=7), dict(out_stride=7), dict(sum_stride=7), dict(out_stride=0), dict(dim=0), dict(dim=65537, xs=65537), dict(dtype=9),
                         dict(sum_dtype=-1), dict(weight_dtype=7), dict(out_type=8), dict(eps=-1e-9), dict(eps=math.nan), dict(eps=math.inf), dict(drop=-0.1), dict(drop=1.0),
                         dict(drop=math.nan), dict(drop=0.999999), dict(scale=7 * P), dict(out_type=rd.RD_E4M3), dict(out_type=rd.RD_E4M3, scale=7 * P + 1),
                         # overlaps: shifted by a row, other strides, each other, the weight, the numbers of the rows
                         dict(out=P + 16), dict(sum=2 * P + 16), dict(out=P, out_stride=16), dict(out=4 * P), dict(out=6 * P), dict(sum=6 * P - 16), dict(rstd=P), dict(rstd=2 * P + 8),
                         dict(rstd=3 * P), dict(rstd=6 * P), dict(out_type=rd.RD_E4M3, scale=5 * P), dict(out_type=rd.RD_E4M3, scale=7 * P, out=P),
                         dict(sum_dtype=rd.RD_FP32, sum=P)],
            [dict(dtype=rd.RD_INT32, sum_dtype=rd.RD_INT32, weight_dtype=rd.RD_INT32), dict(dtype=rd.RD_E4M3, sum_dtype=rd.RD_E4M3, weight_dtype=rd.RD_E4M3), dict(sum_dtype=rd.RD_FP16),
             dict(weight_dtype=rd.RD_FP16), dict(out_type=rd.RD_FP32), dict(n=1 << 31), dict(drop=0.1, first=(1 << 32) - 3), dict(drop=0.1, first=(1 << 64) - 4)])
    assert L.rd_norm(None, P, 8, rd.RD_BF16, None, None, 0, None, None) == rd.RD_ERR_INVALID_ARG
    assert call(**{**good, "n": 0, "x": None, "out": None}) == rd.RD_OK


def test_norm_grad_refusals():
    L, need = rd.lib(), C.c_size_t()
    assert L.rd_norm_grad_workspace(4, 8, C.byref(need)) == rd.RD_OK and need.value == 0          # few rows
    assert L.rd_norm_grad_workspace(1000, 8, C.byref(need)) == rd.RD_OK and need.value >= 32
    assert L.rd_norm_grad_workspace(4, 8, None) == L.rd_norm_grad_workspace(4, 0, C.byref(need)) == L.rd_norm_grad_workspace(4, 65537, C.byref(need)) == rd.RD_ERR_INVALID_ARG
    assert L.rd_norm_grad_workspace(1 << 31, 8, C.byref(need)) == rd.RD_ERR_UNSUPPORTED

    def call(gx, gxs, gr, grs, gw, ws, size, **kw):
        return L.rd_norm_grad(C.byref(rd.rd_norm_grad_t(*kw.values())), gx, gxs, gr, grs, gw, ws, size, None)

    good = dict(gx=5 * P, gxs=8, gr=6 * P, grs=8, gw=7 * P, ws=8 * P, size=need.value, up=P, ups=8, sum=2 * P, ss=8, rstd=3 * P, weight=4 * P, more=9 * P, ms=8, n=1000, dim=8,
                dtype=rd.RD_BF16, sum_dtype=rd.RD_BF16, weight_dtype=rd.RD_BF16, drop=0.0, seed=0, offset=0, first=0)
    refused(call, good, [dict(gx=None, gr=None, gw=None), dict(up=None), dict(sum=None), dict(rstd=None), dict(weight=None), dict(up=P + 1), dict(sum=2 * P + 1), dict(rstd=3 * P + 2),
                         dict(weight=4 * P + 1), dict(gx=5 * P + 1), dict(gr=6 * P + 1), dict(gw=7 * P + 1), dict(more=9 * P + 1), dict(ws=None), dict(ws=8 * P + 128), dict(ups=7),
                         dict(ss=7), dict(ms=7), dict(gxs=7), dict(grs=7), dict(gxs=0), dict(dim=0), dict(dtype=9), dict(drop=1.0), dict(gx=P + 16), dict(gx=6 * P), dict(gr=9 * P + 2),
                         dict(gx=4 * P), dict(gw=4 * P), dict(gw=P), dict(gw=2 * P + 2), dict(gw=9 * P), dict(gr=3 * P), dict(ws=P), dict(ws=2 * P), dict(ws=7 * P), dict(ws=5 * P)],
            [dict(dtype=rd.RD_FP64), dict(sum_dtype=rd.RD_FP16), dict(weight_dtype=rd.RD_INT32), dict(n=1 << 31), dict(drop=0.5, first=1 << 32)])
    assert call(**{**good, "size": need.value - 1}) == rd.RD_ERR_TOO_SMALL
    assert call(**{**good, "n": 0, "up": None, "sum": None, "rstd": None, "gw": None}) == rd.RD_OK


def test_dropout_refusals():
    L = rd.lib()
    good = dict(x=P, xs=8, n=4, dim=8, dtype=rd.RD_BF16, drop=0.5, seed=1, offset=2, first=0, out=2 * P, os=8)
    call = lambda **kw: L.rd_dropout(*kw.values(), None)
    refused(call, good, [dict(x=None), dict(out=None), dict(x=P + 1), dict(out=2 * P + 1), dict(xs=7), dict(os=7), dict(os=0), dict(dim=0), dict(dim=65537, xs=65537, os=65537), dict(dtype=7),
                         dict(drop=1.0), dict(drop=-1.0), dict(drop=math.nan), dict(out=P + 2), dict(out=P, os=9)],
            [dict(dtype=rd.RD_INT64), dict(dtype=rd.RD_E4M3), dict(n=1 << 31), dict(first=1 << 32)])
    assert call(**{**good, "n": 0, "x": None, "out": None}) == rd.RD_OK


@gpu
def test_norm_binding_refusals():
    x, w = torch.zeros(4, 8, device="cuda"), torch.zeros(8, device="cuda")
    r = torch.zeros(4, device="cuda")
    for f in (lambda: rd.rd_norm(x.cpu(), w), lambda: rd.rd_norm(x, w.cpu()), lambda: rd.rd_norm(x, w[:7]), lambda: rd.rd_norm(x.T, w), lambda: rd.rd_norm(x[0], w),
              lambda: rd.rd_norm(x, w, x[:3]), lambda: rd.rd_norm(x, w, x.cpu()), lambda: rd.rd_norm(x, w, out=x[:3]), lambda: rd.rd_norm(x, w, out=x.half()),
              lambda: rd.rd_norm(x, w, x, total=x.half()), lambda: rd.rd_norm(x, w, out_dtype=torch.float16), lambda: rd.rd_norm(x, w, out_dtype=8),
              lambda: rd.rd_norm(x, w, first_row=-1), lambda: rd.rd_norm_grad(x, x[:3], w, r), lambda: rd.rd_norm_grad(x, x, w, r.double()), lambda: rd.rd_norm_grad(x, x, w, r[:3]),
              lambda: rd.rd_norm_grad(x, x, w, r, x.half()), lambda: rd.rd_norm_grad(x, x, w, r, grad_weight=w.half()), lambda: rd.rd_norm_grad(x, x, w, r, grad_x=x.half()),
              lambda: rd.rd_dropout(x, 0.5, 1, out=x[:3]), lambda: rd.rd_dropout(x.cpu(), 0.5, 1)):
        with pytest.raises(ValueError):
            f()
    for f, code in ((lambda: rd.rd_norm(x.double(), w.double()), rd.RD_ERR_UNSUPPORTED), (lambda: rd.rd_norm(x, w.half()), rd.RD_ERR_UNSUPPORTED),
                    (lambda: rd.rd_norm(x, w, drop=1.0), rd.RD_ERR_INVALID_ARG), (lambda: rd.rd_norm(x, w, eps=-1.0), rd.RD_ERR_INVALID_ARG),
                    (lambda: rd.rd_dropout(x, 0.5, 1, first_row=2 ** 32), rd.RD_ERR_UNSUPPORTED)):
        with pytest.raises(rd.RdError) as e:
            f()
        assert e.value.status == code
    with pytest.raises((OverflowError, TypeError)):
        rd.rd_dropout(x, 0.5, -1)
