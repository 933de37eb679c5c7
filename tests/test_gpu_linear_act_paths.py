"""The projection with epilogue on each of its kernels: every size here is
asserted to take the tile that its test is about (lacache_linear_act_tile), for
SwiGLU with the N that gives as many weight rows. The reference and its
tolerance are test_gpu_linear_act's."""

import math
import os
import re

import numpy as np
import pytest
import torch

import paper_2607_16339_amd as lc
from paged_util import DEV
from test_gpu_linear_act import GELU, NONE, SILU, SWIGLU, _case, _check, _want

pytestmark = pytest.mark.gpu

# (weight rows, K, tile's columns, rows): the weight-streaming kernel with one slab of 16
# weight rows (1 to 4 slabs of activations, two passes) and with three
STREAMS = [(2048, 4096, 16, M) for M in (1, 16, 33, 48, 64, 100, 128)] + [(12288, 4096, 48, 20), (12288, 4096, 48, 5)]
# (rows, weight rows, K, tile) of tiles
TILES = [(96, 4096, 2048, (32, 64)), (90, 6144, 2048, (64, 64)), (300, 4352, 512, (64, 128)),
         (1000, 4096, 256, (128, 128)), (2040, 4096, 2048, (128, 256)), (8000, 4096, 1024, (256, 256))]


def _n(rows, act):
    return rows // 2 if act == SWIGLU else rows


def _stream(rows, K, cols, M, act):
    assert lc.lacache_linear_act_tile(M, _n(rows, act), K, act) == (64, cols)
    return M, _n(rows, act), K


def _tile(M, rows, K, tile, act):
    assert lc.lacache_linear_act_tile(M, _n(rows, act), K, act) == tile
    return M, _n(rows, act), K


def _same(x, y):
    return torch.equal(x.view(torch.int16), y.view(torch.int16))


@pytest.mark.parametrize("act", range(6))
@pytest.mark.parametrize("rows,K,cols,M", STREAMS)
def test_residual_updated_in_place_by_the_streaming_kernel(rows, K, cols, M, act):
    size = _stream(rows, K, cols, M, act)
    assert _same(_check(*size, act, True, True, seed=M, in_place=True), _check(*size, act, True, True, seed=M))


def _gelu_bound():
    """The header's bound of GELU's error, relative to |x|."""
    header = os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "include", "lacache.h")
    with open(header) as f:
        return float(re.search(r"off by at most ([0-9.e-]+) \|x\|", f.read()).group(1))


@pytest.mark.parametrize("M", [128, 4096])
def test_gelu_keeps_the_bound_of_the_header(M):
    """x in fp32, a sum of three bf16 parts, and a residual that takes almost all of gelu(x) away
    again: what is left shows the error in front of the rounding. (fp32 steps of the formula: the
    reciprocal's argument and the reciprocal 3 u, which t times the polynomial magnifies by 3.5;
    its four partial sums 3.2 u; two products 2 u; exp2 and its argument 4.6 u; together 20 u of
    erfc, 10 u of its half; the last two operations 1.5 u; the formula's own 1.3 u: 12.8 u = 7.6e-7.)"""
    rng = np.random.default_rng(M)
    x = np.concatenate([rng.uniform(-8.0, 8.0, 1 << 21), rng.uniform(-0.6, 0.6, 1 << 21)]).astype(np.float32)
    x = torch.from_numpy(x)
    y = 0.5 * x.double() * torch.erfc(-x.double() / math.sqrt(2.0))
    x = x[(y - y.to(torch.bfloat16).double()).abs() <= 1e-6 * x.double().abs()]
    x = x[torch.from_numpy(rng.permutation(len(x))[:M])]
    assert len(x) == M
    y = 0.5 * x.double() * torch.erfc(-x.double() / math.sqrt(2.0))
    hi = x.to(torch.bfloat16)
    mid = (x - hi.float()).to(torch.bfloat16)
    lo = (x - hi.float() - mid.float()).to(torch.bfloat16)
    assert torch.equal(hi.double() + mid.double() + lo.double(), x.double())
    a = torch.zeros((M, 128), dtype=torch.bfloat16)
    a[:, 0], a[:, 1], a[:, 2] = hi, mid, lo
    w = torch.zeros((128, 128), dtype=torch.bfloat16)
    w[:, :3] = 1.0
    out = torch.empty((M, 128), dtype=torch.bfloat16, device=DEV)
    # (the sum is x itself)
    r = (-hi)[:, None].expand(M, 128).contiguous().to(DEV)
    lc.lacache_linear_act_bf16(a.to(DEV), w.to(DEV), out, residual=r, act=NONE)
    assert torch.equal(out.cpu().double(), (x.double() - hi.double()).to(torch.bfloat16).double()[:, None].expand(M, 128))
    r = -y.to(torch.bfloat16)
    lc.lacache_linear_act_bf16(a.to(DEV), w.to(DEV), out, residual=r[:, None].expand(M, 128).contiguous().to(DEV), act=GELU)
    left = y + r.double()
    off = ((out.cpu().double() - left[:, None]).abs() - 2.0 ** -8 * left.abs()[:, None]) / x.double().abs()[:, None]
    print("M %d: largest error %.3g |x|" % (M, float(off.max())))
    assert float(off.max()) <= _gelu_bound()
