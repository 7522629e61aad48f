"""Block selection among scores that 32 bits cannot tell apart."""

import numpy as np
import pytest

from oracle import long_context as olc
from paper_2609_33536_amd import workloads
from tests.test_gpu_select import Rows

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,budget", [(500, 77), (500, 250), (60, 13), (3000, 77)])
def test_scores_that_differ_by_a_2_to_the_minus_30_of_their_size(n, budget):
    """2^15 + k 2^-15, k below 250: two or three values in 32 bits."""
    v = np.zeros((1, 1, n, 2, 128), dtype=np.float32)
    v[..., 1, 0] = 2.0 ** 15
    v[0, 0, :, 1, 1] = np.random.default_rng(1).permutation(n) % 250 * 2.0 ** -15   # (fits 8 bits)
    q = workloads.to_words(np.ones((1, 1, 128), dtype=np.float32), "bf16")
    words = workloads.to_words(v, "bf16")
    x = olc.values(words, "bf16")
    assert np.array_equal(x, v)
    scores = olc.scores(np.ones((1, 128)), x[0, 0, :, 0], x[0, 0, :, 1])
    assert len(np.unique(scores)) == min(n, 250) and len(np.unique(scores.astype(np.float32))) <= 3
    Rows([16 * n], 1, 1, bounds=words, q=q).check(budget, 0, 0)
