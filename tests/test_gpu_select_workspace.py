"""Block selection on one workspace that was made for the largest batch, as sequences end and
shorter ones come: the lists against the oracle, no byte behind the workspace written."""

import numpy as np
import pytest

from paper_2609_33536_amd import ekv
from tests.gpu_util import require_gpu
from tests.test_gpu_select import Rows

pytestmark = pytest.mark.gpu
CANARY = 4096


@pytest.mark.parametrize("dtype", ["bf16", "e5m2"])
def test_one_workspace_for_a_batch_that_shrinks(dtype):
    torch = require_gpu()
    budget, memory = 64, None
    rng = np.random.default_rng(1)
    for batch, blocks in ((33, 1300), (32, 1300), (16, 1300), (9, 700), (4, 1300), (1, 1299), (1, 65), (2, 600)):
        lens = 16 * rng.integers(blocks // 2, blocks + 1, size=batch)
        lens[0] = 16 * blocks
        r = Rows(lens, 4, 4, dtype, seed=blocks + batch)
        if memory is None:
            size = ekv.select_workspace_bytes(r.pool, r.batch, budget)
            memory = torch.full((size + CANARY,), 0xA5, dtype=torch.uint8, device="cuda")
        r.check(budget, 1, 2, ws=memory[:size])
        r.check(7, 0, 0, ws=memory[:size])
        assert bool((memory[size:] == 0xA5).all())
