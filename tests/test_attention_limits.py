"""Scales that block attention refuses, with nothing launched (CPU)."""
import pytest

from test_decode_abi import attend


@pytest.mark.parametrize("scale", [(1 + 2.0 ** -23) * 2.0 ** 127, -1.25 * 2.0 ** 127, (2 - 2.0 ** -23) * 2.0 ** 127])
def test_scales_that_overflow_with_the_logarithm_are_refused(scale):
    assert attend(scale=scale) == 1
