"""The EKV_DEBUG=1 checks of the serving step: a free list that names a block twice or
one in use, and a token slot given to two rows, are refused before anything is enqueued."""

import numpy as np
import pytest

from paper_2609_33536_amd import ekv
from tests.gpu_util import require_gpu

pytestmark = pytest.mark.gpu


def _extension(ids, head, count, lens=(20, 0), table=((0, 1, 9, 9), (9, 9, 9, 9)), num_blocks=16):
    torch = require_gpu()
    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    st = dict(ids=i32(ids), cursor=i32([head, count]), lens=i32(lens), table=i32(table), cu=i32([0] * 3), slots=i32([0] * 40),
              status=i32([9] * 4), out=i32([9] * 2), cursor_out=i32([9, 9]))
    ekv.extend(ekv.make_free_list(st["ids"], st["cursor"], num_blocks, st["cursor_out"]), st["lens"], i32([13, 3]), st["table"], None,
               st["out"], st["cu"], st["slots"], None, st["status"])
    torch.cuda.synchronize()
    return st


@pytest.mark.parametrize("ids,head,count,word", [
    ([4, 5, 6, 5], 0, 4, "twice"), ([5, 4, 6, 5], 3, 2, "twice"), ([4, 1, 6, 7], 0, 3, "held by sequence 0"),
    ([1, 4, 6, 0], 3, 2, "held by sequence 0")])
def test_free_lists_that_name_a_block_twice_or_one_in_use(ids, head, count, word, monkeypatch):
    monkeypatch.setenv("EKV_DEBUG", "1")
    with pytest.raises(ekv.EkvError, match=word) as e:
        _extension(ids, head, count)
    assert e.value.status == ekv.ERR_INVALID


@pytest.mark.parametrize("ids,head,count", [
    ([4, 5, 6, 5], 0, 3),          # (the second 5 is no longer in the list)
    ([1, 4, 5, 0], 1, 2),          # (nor are the blocks in use)
    ([4, 9, 6, 7], 0, 4),          # 9: in the table, but in no row's length
    ([4, 99, -1, 99], 0, 4),       # outside the pool: no slot, no reason
    ([4, 5, 6, 7], -3, 99)])       # a cursor outside its ring is brought into it
def test_valid_free_lists_extend_as_without_the_checks(ids, head, count, monkeypatch):
    want = _extension(ids, head, count)
    monkeypatch.setenv("EKV_DEBUG", "1")
    got = _extension(ids, head, count)
    for name in want:
        assert (want[name] == got[name]).all(), name


@pytest.mark.parametrize("slots,word", [([3, 17, 3], "slot 3 for two rows"), ([40, 40, -1], "slot 40 for two rows"), ([5, -1, -1], None),
                                        ([64, 64, 0], None), ([2**31 - 1, 1, 2], None)])
def test_slots_given_to_two_rows(slots, word, monkeypatch):
    torch = require_gpu()
    kv = torch.zeros((4, 2, 1, 16, 128), dtype=torch.int16, device="cuda")   # slots 0 .. 63
    pool = ekv.make_pool(kv, 1)
    turns = torch.from_numpy(ekv.rope_freqs(64).view(np.int64)).cuda()
    x = torch.ones((3, 1, 128), dtype=torch.bfloat16, device="cuda")
    q = torch.zeros_like(x)
    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    call = lambda: ekv.rope_append(pool, ekv.make_rope(turns, 64), i32([0, 1, 2]), i32(slots), x, x, x, q)  # noqa: E731
    monkeypatch.setenv("EKV_DEBUG", "1")
    if word is None:
        call()
        torch.cuda.synchronize()
        assert q.any()
        return
    with pytest.raises(ekv.EkvError, match=word):
        call()
    torch.cuda.synchronize()
    assert not kv.any() and not q.any()
