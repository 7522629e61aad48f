"""PagedKV.extend without a GPU: a call that raises at any step leaves the mirror
as it was, so that mirror and device never part."""

import numpy as np
import pytest

from paper_2609_33536_amd import ekv, kvpool

torch = pytest.importorskip("torch")


class _Kv(kvpool.PagedKV):
    """The state of a PagedKV over CPU tensors; uploads are plain copies."""

    def __init__(self, seq_lens, width=4, free=(7, 8, 9), tags=None):
        table = np.arange(len(seq_lens) * width, dtype=np.int32).reshape(-1, width) + 100
        self.mirror = kvpool.HostMirror(table, seq_lens, 64, free, tags)
        self.bt, self.tags, self.seq_lens = (torch.from_numpy(a.copy()) for a in (self.mirror.bt, self.mirror.tags, self.mirror.seq_lens))
        self.device = "cpu"

    def _upload(self, arr):
        return torch.from_numpy(np.ascontiguousarray(arr))


def _state(m):
    return m.bt.tolist(), m.tags.tolist(), m.seq_lens.tolist(), list(m.free)


@pytest.fixture
def kv():
    return _Kv([0, 20])


@pytest.mark.parametrize("start", [torch.tensor([0, 5]), torch.tensor([0, 5, 6], dtype=torch.int32),
                                   torch.tensor([0.0, 5.0]), torch.tensor([[0, 5]], dtype=torch.int32),
                                   torch.tensor([0, 5], dtype=torch.int32)],   # (the last one: host memory)
                         ids=["int64", "length", "float", "shape", "host"])
def test_a_start_that_is_refused_leaves_the_mirror(kv, start):
    before = _state(kv.mirror)
    with pytest.raises(ekv.EkvError, match="start|GPU tensor") as e:
        kv.extend([3, 20], start)
    assert e.value.status == ekv.ERR_INVALID
    assert _state(kv.mirror) == before


@pytest.mark.parametrize("step", ["upload", "memory", "launch"])
def test_a_step_that_fails_leaves_the_mirror(kv, step, monkeypatch):
    def fail(*a, **k):
        raise RuntimeError("out of memory")
    before = _state(kv.mirror)
    if step == "upload":
        monkeypatch.setattr(kv, "_upload", fail)
    elif step == "memory":
        monkeypatch.setattr(torch, "empty", fail)
    else:
        monkeypatch.setattr(ekv, "make_free_list", lambda *a: None)
        monkeypatch.setattr(ekv, "extend", fail)
    with pytest.raises(RuntimeError):
        kv.extend([3, 20])
    assert _state(kv.mirror) == before


def test_the_mirror_follows_the_launch(kv, monkeypatch):
    """The call's arguments are those of the extension that the mirror then shows."""
    seen = {}
    monkeypatch.setattr(ekv, "make_free_list", lambda ids, cursor, blocks: seen.update(ids=ids.tolist(), cursor=cursor.tolist()))

    def launch(free, lens, new, *rest):
        seen.update(lens=lens.tolist(), new=new.tolist(), mirror=_state(kv.mirror))
    monkeypatch.setattr(ekv, "extend", launch)
    before = _state(kv.mirror)
    kv.extend([3, 20])
    assert seen["mirror"] == before and seen["lens"] == [0, 20] and seen["new"] == [3, 20]
    assert seen["ids"][:2] == [7, 8] and seen["cursor"] == [0, 2]
    assert kv.mirror.seq_lens.tolist() == [3, 40] and list(kv.mirror.free) == [9]
    assert kv.mirror.bt[0, 0] == 7 and kv.mirror.bt[1, 2] == 8


def test_new_tokens_never_go_into_a_base_block():
    """The device takes nothing where a partly filled block is tagged BASE: neither does the mirror."""
    tags = np.zeros((3, 4), dtype=np.uint8)
    tags[:, 1] = 1
    m = kvpool.HostMirror(np.arange(12).reshape(3, 4), [32, 20, 0], 64, [20, 21, 22], tags)
    before = _state(m)
    with pytest.raises(ekv.EkvError, match="BASE") as e:
        m.plan_extend([0, 1, 1])
    assert e.value.status == ekv.ERR_INVALID and _state(m) == before
    assert m.plan_extend([1, 0, 1]).tolist() == [20, 21]   # (full BASE blocks, and rows that do not grow, are no reason)


def test_what_the_device_refused_is_there_to_read(kv, monkeypatch):
    """The status of the last extension is kept on the device; with EKV_DEBUG=1 a refusal raises and the mirror
    stays, as the device did."""
    def launch(free, lens, new, bt, tags, out, cu, slots, pos, status, *rest):
        status.copy_(torch.tensor(reply, dtype=torch.int32))
    monkeypatch.setattr(ekv, "make_free_list", lambda *a: None)
    monkeypatch.setattr(ekv, "extend", launch)
    before, reply = _state(kv.mirror), [ekv.EXTEND_ROW, 0, 0, 2]
    monkeypatch.setenv("EKV_DEBUG", "1")
    with pytest.raises(ekv.EkvError, match="took nothing"):
        kv.extend([3, 20])
    assert _state(kv.mirror) == before
    reply = [0, 23, 2, 0]
    kv.extend([3, 20])
    assert kv.extend_status.tolist() == reply and kv.mirror.seq_lens.tolist() == [3, 40]


@pytest.mark.parametrize("b", [1, 2, 3, 4])
@pytest.mark.parametrize("new", [0, 1, 3, 4, 45])
def test_slots_and_positions_are_aligned_for_the_wide_stores(b, new, monkeypatch):
    kv, seen = _Kv([0] * b, free=range(20)), {}
    monkeypatch.setattr(ekv, "make_free_list", lambda *a: None)
    monkeypatch.setattr(ekv, "extend", lambda free, lens, n, bt, tags, out, cu, slots, pos, status, *rest: seen.update(
        slots=slots, pos=pos, cu=cu, status=status))
    cu, slots, positions = kv.extend([new] * b)
    assert slots is seen["slots"] and positions is seen["pos"] and cu is seen["cu"]
    assert slots.numel() == positions.numel() == b * new and cu.numel() == b + 1 and seen["status"].numel() == 4
    spans = []
    for t in (slots, positions, cu, seen["status"]):
        if t.numel():
            spans.append((t.data_ptr(), t.data_ptr() + 4 * t.numel()))
    for t in (slots, positions):
        assert t.numel() == 0 or t.data_ptr() % 16 == 0
    spans.sort()
    assert all(a[1] <= c[0] for a, c in zip(spans, spans[1:]))
