"""Decode over selected blocks at the edges of its workspace."""

import pytest

from paper_2609_33536_amd import ekv
from tests.gpu_util import default_scale, require_gpu
from tests.test_gpu_decode_selected import _check, _decode, _lists, _repeated

pytestmark = pytest.mark.gpu
CANARY = 4096
COUNTERS = 32768


@pytest.mark.parametrize("dtype", ["bf16", "e5m2"])
@pytest.mark.parametrize("batch,hkv,hq,budget", [(1, 1, 16, 1000), (2, 8, 32, 200), (16, 8, 8, 130), (40, 8, 64, 130)])
def test_workspaces_smaller_than_the_reported_size(batch, hkv, hq, budget, dtype):
    """Down to the merge counters alone: lists in fewer pieces, nothing written behind the workspace."""
    torch = require_gpu()
    c = _repeated(batch, 520, hq, hkv, dtype, seed=budget)
    selected, counts = _lists(c, budget, 1)
    need = ekv.decode_selected_workspace_bytes(c.kv.pool, c.batch, budget)
    assert need > COUNTERS
    for size in sorted({COUNTERS, COUNTERS + 8, (COUNTERS + need) // 2 + 3, need - 1, need}):
        print(f"selected: B={batch} Hq={hq} Hkv={hkv} budget={budget} {dtype} workspace {size} of {need}", flush=True)
        memory = torch.zeros(size + CANARY, dtype=torch.uint8, device="cuda")
        memory[size:] = 0xA5
        for _ in range(2):
            _check(c, selected, counts, _decode(c, selected, counts, ws=memory[:size]), default_scale())
        assert bool((memory[size:] == 0xA5).all()) and not memory[:COUNTERS].any()


def test_one_workspace_for_a_batch_that_shrinks():
    """Made for the largest batch: 70 sequences need no partial results, fewer of them do."""
    budget = 150
    big = _repeated(70, 300, 32, 8, "bf16", seed=1)
    ws = ekv.decode_selected_workspace(big.kv.pool, big.batch, budget)
    for batch in (70, 48, 33, 17, 16, 5, 1):
        c = _repeated(batch, 300, 32, 8, "bf16", seed=batch)
        selected, counts = _lists(c, budget, batch)
        print(f"selected: {batch} sequences on a workspace of {ws.numel()}", flush=True)
        _check(c, selected, counts, _decode(c, selected, counts, ws=ws), default_scale())
