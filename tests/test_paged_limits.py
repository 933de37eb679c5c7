"""Sizes and numbers at the ends of what the paged cache's calls and the
projection with epilogue take, on the host: fake, aligned, non-overlapping
addresses that are never dereferenced (every call here is refused)."""

import ctypes

import pytest

from test_paged_abi import INVALID, OK, L, UNSUP, _attn, _linear  # noqa: F401


@pytest.mark.parametrize("scale", [2.4e38, 3.0e38, 3.4e38])
def test_scale_whose_factor_in_base_2_is_infinite(L, scale):  # noqa: F811
    """A score of 0 times that factor would be no number. (2.4e38 log2(e) is above 3.4e38.)"""
    assert _attn(L, scale=scale) == INVALID
    assert _attn(L, S=0, scale=scale) == INVALID


@pytest.mark.parametrize("sizes", [dict(M=1 << 24, N=8192), dict(M=1 << 24, N=131072), dict(M=1 << 24, N=4096, act=5)])
def test_projection_whose_launch_would_count_too_many_threads(L, sizes):  # noqa: F811
    """2^17 x 32 tiles of 128 x 256 on 16 wavefronts are 2^32 threads (the output, 256 GiB, fits the memory)."""
    assert _linear(L, K=128, out=1 << 50, bias=None, residual=None, **sizes) == UNSUP


def test_hook_of_the_projections_wavefronts(L):  # noqa: F811
    waves = ctypes.c_int()
    assert L.lacache_linear_act_waves(300, 256, 128, 0, ctypes.byref(waves)) == OK and waves.value in (4, 8, 16)
    for bad in ((0, 256, 128, 0), (-1, 256, 128, 0), (300, 100, 128, 0), (300, 256, 64, 0), (300, 256, 128, 6)):
        assert L.lacache_linear_act_waves(*bad, ctypes.byref(waves)) == INVALID, bad
    assert L.lacache_linear_act_waves(300, 256, 128, 0, None) == INVALID
    assert L.lacache_linear_act_waves(300, 131072 + 128, 128, 0, ctypes.byref(waves)) == UNSUP
