"""Calls of the cache operators that are refused for what their arguments mean together, without a GPU."""
import math

import pytest

from test_cache_ops import attend, blocks


@pytest.mark.parametrize("sparse", [False, True])
@pytest.mark.parametrize("scale", [3e38, -3e38, 3.4028234e38, math.inf, -math.inf, math.nan])
def test_scales_without_a_finite_power_of_two(scale, sparse):
    """Weights are powers of two: scale * log2(e) has to be a number of 32 bits, too."""
    assert attend(scale=scale, blocks=blocks() if sparse else None) == -1
