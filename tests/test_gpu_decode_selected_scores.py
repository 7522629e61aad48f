"""Decode over selected blocks of scores at the end of the 32-bit range."""

import numpy as np
import pytest

from oracle import long_context as olc
from tests.context_util import Cache
from tests.gpu_util import require_gpu, words_to_tensor
from tests.test_gpu_decode_selected import _decode

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("budget", [10, 40])
def test_equal_scores_next_to_the_lowest_float(budget):
    """Every score -2^127 scale log2(e) = -3.19 10^38, above the lowest float: each token weighs the same, and the result is
    the mean of V.  Powers of zero are exactly 1 and the weights' sum is exact, so that the sum over n tokens and the division
    are off by (n + 3) 2^-24 of the sizes; V in halves adds nothing (weights of 1)."""
    torch = require_gpu()
    c = Cache([16 * budget - 3], 4, 2, seed=budget)
    c.q_words[:] = 0
    c.q_words[0, :, 0] = 0x3F80      # 1.0
    c.q = words_to_tensor(c.q_words, torch, "bf16")
    c.pool[:, 0, :, :, 0] = 0xFF00   # -2^127
    c.kv.kv.copy_(torch.from_numpy(c.pool.view(np.int16)).cuda().view(c.kv.kv.dtype).view(c.kv.kv.shape))
    every = np.broadcast_to(np.arange(budget, dtype=np.int32), (1, 2, budget)).copy()
    out = _decode(c, every, np.full((1, 2), budget), scale=1.3)
    for h in range(2):
        _, v = olc.listed_tokens(c.pool, c.bt[0], c.tags[0], c.lens[0], every[0, h], h, "bf16")
        off = np.abs(out[0, 2 * h:2 * h + 2] - v.mean(axis=0))
        assert (off <= (len(v) + 3) * 2.0 ** -24 * np.abs(v).mean(axis=0)).all()
