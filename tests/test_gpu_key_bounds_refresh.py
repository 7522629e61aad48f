"""Key bounds of one cache through transitions: bounds that are there, pairs demoted and
refined in place, and the blocks from the first changed pair on refreshed."""

import numpy as np
import pytest

from oracle import fp8 as ofp8
from oracle import long_context as olc
from oracle import transitions as otr
from paper_2609_33536_amd import ekv
from tests.context_util import Cache
from tests.gpu_util import require_gpu

pytestmark = pytest.mark.gpu
PAIRS = np.array([[0, 1], [0, 3], [2, 0], [2, 20], [2, 19]], dtype=np.int32)


def _refresh(c, bounds, known):
    """The bounds from known on, in place; the others are as they were."""
    torch = require_gpu()
    elem = c.pool.dtype
    old = bounds.cpu().numpy().view(elem)
    ekv.key_bounds(c.kv.pool, c.batch, bounds, torch.tensor(known, dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    got = bounds.cpu().numpy().view(elem)
    assert np.array_equal(got, olc.bounds(c.pool, c.bt, c.tags, c.lens, known, old, c.dtype))
    fresh = olc.bounds(c.pool, c.bt, c.tags, c.lens, [0] * len(c.lens), old, c.dtype)
    assert np.array_equal(got, fresh)   # (nothing before the first changed pair is stale)
    return got


def _lower(c, structured):
    mode = c.kv.relower()
    if mode != ekv.MODE_NATIVE and not structured:
        mode = ekv.MODE_GENERAL
    c.batch = ekv.make_batch(c.kv.seq_lens, c.kv.bt, c.kv.tags, c.kv.bounds if structured else None, c.hq, mode, int(c.lens.max()))


@pytest.mark.parametrize("structured", [True, False])
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "e5m2"])
def test_refresh_after_a_demotion_and_a_refinement(dtype, structured):
    oracle = ofp8 if dtype == "e5m2" else otr
    c = Cache([130, 64, 700], 8, 2, dtype=dtype, seed=8, spare=4, structured=structured)
    bounds = ekv.key_bounds_buffer(c.kv.pool, c.batch)
    target = _refresh(c, bounds, [0, 0, 0])

    freed, lo, _ = c.kv.demote(PAIRS)
    c.kv.commit()
    c.pool, c.bt, c.tags, want_freed, want_lo = oracle.demote(c.pool, c.bt, c.tags, PAIRS, c.lens)
    assert np.array_equal(c.kv.bt.cpu().numpy(), c.bt)
    _lower(c, structured)
    # (sequence 0 from its first demoted pair on, inside its second block; sequence 1 nothing; sequence 2 whole)
    base = _refresh(c, bounds, [32, 64, 0])
    changed = (base != target).any(axis=(1, 3, 4))
    assert changed[0].nonzero()[0].tolist() == [2, 3, 6, 7] and not changed[1].any()
    assert changed[2].nonzero()[0].tolist() == [0, 1, 38, 39, 40, 41]

    # a refinement of some of them: those are as they were, the others BASE still
    some = [0, 3, 4]
    new = c.kv.refine(PAIRS[some], lo[some].contiguous())
    c.pool, c.bt, c.tags = oracle.refine(c.pool, c.bt, c.tags, PAIRS[some], new, want_lo[some], c.lens)
    _lower(c, structured)
    got = _refresh(c, bounds, [40, 64, 16 * 38 + 15])
    changed = (got != target).any(axis=(1, 3, 4))
    assert changed[0].nonzero()[0].tolist() == [6, 7] and changed[2].nonzero()[0].tolist() == [0, 1]

    rest = [1, 2]
    new = c.kv.refine(PAIRS[rest], lo[rest].contiguous())
    c.pool, c.bt, c.tags = oracle.refine(c.pool, c.bt, c.tags, PAIRS[rest], new, want_lo[rest], c.lens)
    _lower(c, structured)
    assert np.array_equal(_refresh(c, bounds, [96, 64, 0]), target)
