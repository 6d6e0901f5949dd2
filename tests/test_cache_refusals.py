"""Calls of the cache operators that are refused for what their arguments mean together, without a GPU."""
import math

import pytest

from paper_1811_03115_amd import binding
from test_cache_ops import P, attend, blocks


@pytest.mark.parametrize("sparse", [False, True])
@pytest.mark.parametrize("scale", [3e38, -3e38, 3.4028234e38, math.inf, -math.inf, math.nan])
def test_scales_without_a_finite_power_of_two(scale, sparse):
    """Weights are powers of two: scale * log2(e) has to be a number of 32 bits, too."""
    assert attend(scale=scale, blocks=blocks() if sparse else None) == -1


def test_results_of_a_verification_over_each_other():
    """Four results in three places hold none of them."""
    L = binding.lib()
    far = [P * (i + 1) for i in range(10)]

    def accept(b=3, t=4, **kw):
        a = dict(zip(("path", "accepted", "next", "new_length"), far[6:])) | kw
        return L.bpd_tree_accept(*far[:6], 2, b, t, a["path"], a["accepted"], a["next"], a["new_length"], None, None)

    for kw in (dict(accepted=far[8]), dict(next=far[9]), dict(new_length=far[7] + 8), dict(accepted=far[6] + 44), dict(path=far[8] - 44), dict(path=far[9])):
        assert accept(**kw) == -1, kw
        assert binding.lib().bpd_op_error()
