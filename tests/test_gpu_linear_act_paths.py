"""The projection with epilogue on each of its kernels: every size here is
asserted to take the tile that its test is about (lacache_linear_act_tile), for
SwiGLU with the N that gives as many weight rows. The reference and its
tolerance are test_gpu_linear_act's."""

import math

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
