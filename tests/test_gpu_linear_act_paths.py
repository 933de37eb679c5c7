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
from test_gpu_linear_act import GELU, NONE, SWIGLU, _case, _check

pytestmark = pytest.mark.gpu

# (weight rows, K, tile's columns, rows): the weight-streaming kernel with one slab of 16
# weight rows (1 to 4 slabs of activations, two passes) and with three
STREAMS = [(2048, 4096, 16, M) for M in (1, 16, 33, 48, 64, 100, 128)] + [(12288, 4096, 48, 20), (12288, 4096, 48, 5)]
# (rows, weight rows, K, tile, wavefronts) of tiles
TILES = [(96, 4096, 2048, (32, 64), 4), (90, 6144, 2048, (64, 64), 8), (300, 4352, 512, (64, 128), 8),
         (1000, 4096, 256, (128, 128), 16), (2040, 4096, 384, (128, 256), 16), (2040, 4096, 2048, (128, 256), 8),
         (8000, 4096, 1024, (256, 256), 8)]


def _n(rows, act):
    return rows // 2 if act == SWIGLU else rows


def _stream(rows, K, cols, M, act):
    assert lc.lacache_linear_act_tile(M, _n(rows, act), K, act) == (64, cols)
    assert lc.lacache_linear_act_waves(M, _n(rows, act), K, act) == 4
    return M, _n(rows, act), K


def _tile(M, rows, K, tile, waves, act):
    assert lc.lacache_linear_act_tile(M, _n(rows, act), K, act) == tile
    assert lc.lacache_linear_act_waves(M, _n(rows, act), K, act) == waves
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


@pytest.mark.parametrize("act", range(6))
@pytest.mark.parametrize("bias,residual", [(False, False), (True, False), (False, True)])
@pytest.mark.parametrize("rows,K,cols,M", STREAMS)
def test_optional_operands_of_the_streaming_kernel(rows, K, cols, M, bias, residual, act):
    _check(*_stream(rows, K, cols, M, act), act, bias, residual, seed=M + 1)


@pytest.mark.parametrize("act", range(6))
@pytest.mark.parametrize("bias,residual,in_place", [(True, True, False), (True, True, True), (False, True, False), (True, False, False)])
@pytest.mark.parametrize("M,rows,K,tile,waves", TILES)
def test_operands_of_every_tile(M, rows, K, tile, waves, bias, residual, in_place, act):
    _check(*_tile(M, rows, K, tile, waves, act), act, bias, residual, seed=M + 2, in_place=in_place)


def _far(M, N, K, act):
    """Sums of hundreds, where exp overflows, and a bias that is no number in three columns."""
    _check(M, N, K, act, True, False, seed=9, std=300.0 / math.sqrt(K / 256))
    a, w, b, r = _case(M, N, K, act, True, True, seed=10)
    clean = torch.empty((M, N), dtype=torch.bfloat16, device=DEV)
    lc.lacache_linear_act_bf16(a, w, clean, bias=b, residual=r, act=act)
    b[0], b[1], b[2] = math.inf, -math.inf, math.nan
    if act == SWIGLU:
        b[N + 3], b[N + 4] = math.inf, math.nan  # of the up rows
    out = torch.empty_like(clean)
    lc.lacache_linear_act_bf16(a, w, out, bias=b, residual=r, act=act)
    torch.cuda.synchronize()
    o = out.float()
    assert bool((o[:, 0].abs() == math.inf).all())
    assert bool(torch.isnan(o[:, 2]).all()) and bool((out[:, 2].view(torch.int16) == 0x7FC0).all())
    if act == NONE:
        assert bool((o[:, 1] == -math.inf).all())
    first = 3
    if act == SWIGLU:
        first = 5
        assert bool((o[:, 3].abs() == math.inf).all()) and bool((out[:, 4].view(torch.int16) == 0x7FC0).all())
    assert _same(out[:, first:], clean[:, first:])  # and nothing else moves


@pytest.mark.parametrize("act", range(6))
@pytest.mark.parametrize("rows,K,cols,M", STREAMS)
def test_far_arguments_of_the_streaming_kernel(rows, K, cols, M, act):
    _far(*_stream(rows, K, cols, M, act), act)


@pytest.mark.parametrize("act", range(6))
@pytest.mark.parametrize("M,rows,K,tile,waves", TILES)
def test_far_arguments_of_every_tile(M, rows, K, tile, waves, act):
    _far(*_tile(M, rows, K, tile, waves, act), act)


@pytest.mark.parametrize("act", [GELU, SWIGLU])
@pytest.mark.parametrize("size", [_stream] + [_tile], ids=["stream", "tiles"])
def test_captured_and_replayed_on_every_kernel(size, act):
    for args in (STREAMS if size is _stream else TILES):
        M, N, K = size(*args, act)
        a, w, b, r = _case(M, N, K, act, True, True, seed=11)
        out = torch.empty((M, N), dtype=torch.bfloat16, device=DEV)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            lc.lacache_linear_act_bf16(a, w, out, bias=b, residual=r, act=act)
        for k in range(3):
            a.mul_(-0.5)
            graph.replay()
            torch.cuda.synchronize()
            got = out.clone()
            lc.lacache_linear_act_bf16(a, w, out, bias=b, residual=r, act=act)
            torch.cuda.synchronize()
            assert _same(got, out), (args, k)
