"""Sizes and numbers at the ends of what the paged cache's calls and the
projection with epilogue take, on the host: fake, aligned, non-overlapping
addresses that are never dereferenced (every call here is refused)."""

import pytest

from test_paged_abi import INVALID, L, _attn  # noqa: F401


@pytest.mark.parametrize("scale", [2.4e38, 3.0e38, 3.4e38])
def test_scale_whose_factor_in_base_2_is_infinite(L, scale):  # noqa: F811
    """A score of 0 times that factor would be no number. (2.4e38 log2(e) is above 3.4e38.)"""
    assert _attn(L, scale=scale) == INVALID
    assert _attn(L, S=0, scale=scale) == INVALID
