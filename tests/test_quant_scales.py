"""Scales that a cache of e4m3 codes may have: powers of two, since kernels read the exponent of some of them alone.  No GPU needed."""
import math

import pytest
import torch

from paper_2603_08026_amd import binding as B


def _cache(codes, value, which=0):
    c = [torch.zeros(2, 5, 3, 64, dtype=torch.int8).view(codes) for _ in range(2)]
    s = [torch.ones(2, 3, 5) for _ in range(2)]
    s[which][1, 2, 3] = value
    return B.QuantCache(*c, *s)


@pytest.mark.parametrize("which", [0, 1])
@pytest.mark.parametrize("value", [1.0, 0.0, 2.0 ** -100, 2.0 ** -126, 2.0 ** 119, 0.5, math.nan])
def test_powers_of_two_are_taken(value, which):
    _cache(torch.float8_e4m3fn, value, which)


@pytest.mark.parametrize("which", [0, 1])
@pytest.mark.parametrize("value", [0.3, 1 + 2.0 ** -23, 448.0, -1.0, -0.0, math.inf, -math.inf, 2.0 ** -130, 1.0 / 448])
def test_others_are_refused(value, which):
    with pytest.raises(ValueError, match="powers of two"):
        _cache(torch.float8_e4m3fn, value, which)


@pytest.mark.parametrize("value", [0.3, 1.0 / 127, 2.0 ** -100 / 127, math.nan, 0.0])
def test_int8_takes_any(value):
    _cache(torch.int8, value)


def test_an_empty_cache_is_one_of_zeros():
    c = B.QuantCache.empty(2, 5, 3, 64, device="cpu")
    assert not c.k_scale.any() and not c.v_scale.any() and c.format == B.E4M3
