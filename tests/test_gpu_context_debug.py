"""EKV_DEBUG=1 of the long-context calls: invalid metadata and lists that name a
block twice are refused with nothing enqueued."""

import numpy as np
import pytest

from paper_2609_33536_amd import ekv
from tests.context_util import Cache
from tests.gpu_util import default_scale, require_gpu

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def debug(monkeypatch):
    monkeypatch.setenv("EKV_DEBUG", "1")


def _calls(c, selected, counts=None):
    torch = require_gpu()
    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    bounds = ekv.key_bounds_buffer(c.kv.pool, c.batch)
    sel, out = i32(selected), torch.full(c.q.shape, 7.0, device="cuda")
    picked, n = torch.full_like(sel, 7), torch.full(sel.shape[:2], 7, dtype=torch.int32, device="cuda")
    ws = ekv.select_workspace(c.kv.pool, c.batch, sel.shape[2]), ekv.decode_selected_workspace(c.kv.pool, c.batch, sel.shape[2])
    bounds.fill_(7)
    return dict(bounds=(bounds, lambda: ekv.key_bounds(c.kv.pool, c.batch, bounds)),
                select=(picked, lambda: ekv.select_blocks(c.kv.pool, c.batch, c.q, bounds, picked, n, ws[0])),
                decode=(out, lambda: ekv.attn_decode_selected(c.kv.pool, c.batch, sel, None if counts is None else i32(counts), c.q, out,
                                                              default_scale(), ws[1])))


def test_valid_calls_run():
    c = Cache([100, 40, 0], 8, 2, base=0.5, seed=1)
    torch = require_gpu()
    for out, call in _calls(c, [[[0, 2, -1, -1, 6]] * 2] * 3).values():
        call()
        torch.cuda.synchronize()
        assert (out != 7).any()


def test_bad_metadata_is_refused():
    torch = require_gpu()
    c = Cache([100, 40, 0], 8, 2, seed=2)
    c.kv.bt[1, 1] = 10 ** 6
    for out, call in _calls(c, [[[0, 2]] * 2] * 3).values():
        with pytest.raises(ekv.EkvError, match="EKV_DEBUG"):
            call()
        torch.cuda.synchronize()
        assert (out == 7).all()


@pytest.mark.parametrize("selected,counts,refused", [
    ([0, 2, 2, 5], None, True), ([3, 0, 5, 3], None, True), ([3, 0, 5, 3], 3, False), ([-1, 4, -1, 9], None, False),
    ([99, 1, 99, 2], None, False), ([9, 1, 99, 9], None, True), ([1, 1, 0, 0], 1, False), ([1, 1, 0, 0], 100, True), ([1, 1, 0, 0], -4, False)])
def test_blocks_listed_twice_are_refused(selected, counts, refused):
    torch = require_gpu()
    c = Cache([100, 160], 8, 2, seed=3)
    lists = np.tile(np.arange(4), (2, 2, 1))
    lists[1, 1] = selected
    n = None if counts is None else [[4, 4], [4, counts]]
    out, call = _calls(c, lists.tolist(), n)["decode"]
    if refused:
        with pytest.raises(ekv.EkvError, match="listed twice for sequence 1, KV head 1"):
            call()
    else:
        call()
    torch.cuda.synchronize()
    assert (out == 7).all() == refused
