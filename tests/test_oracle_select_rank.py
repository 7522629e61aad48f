"""The selection oracle's order of scores that are infinite or no numbers."""

import numpy as np
import pytest

from oracle import long_context as olc

INF, NAN = 0x7F80, 0x7FC0   # bf16


def _pick(high, budget):
    b = np.zeros((1, 1, len(high), 2, 128), dtype=np.uint16)
    b[0, 0, :, 1, 0] = high
    q = np.zeros((1, 1, 128))
    q[..., 0] = 1.0
    return olc.select(q, b, [16 * len(high)], budget, 0, 0, "bf16")[0][0, 0].tolist()


@pytest.mark.parametrize("budget,want", [(1, [3]), (2, [3, 5]), (3, [0, 3, 5]), (4, [0, 2, 3, 5]), (5, [0, 2, 3, 4, 5])])
def test_what_is_no_number_comes_before_infinity(budget, want):
    """inf, 1, inf, NaN, 2, -NaN, -inf"""
    assert _pick([INF, 0x3F80, INF, NAN, 0x4000, NAN | 0x8000, INF | 0x8000], budget) == want


def test_a_query_that_is_no_number_leaves_the_first_blocks():
    b = np.zeros((1, 1, 6, 2, 128), dtype=np.uint16)
    b[0, 0, :, 1, 0] = [0, 0x3F80, 0x4000, 0x3F80, INF, 0]
    q = np.ones((1, 2, 128))
    q[0, 1, 9] = np.nan
    assert olc.select(q, b, [96], 3, 0, 1, "bf16")[0][0, 0].tolist() == [0, 1, 5]
