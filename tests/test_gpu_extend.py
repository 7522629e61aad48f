"""Table extension on the GPU against the plain oracle: whole numbers, exact,
with every array's neighbours left as they were."""

import numpy as np
import pytest

from oracle import serve
from paper_2609_33536_amd import ekv, kvpool, workloads
from tests.gpu_util import require_gpu

pytestmark = pytest.mark.gpu
CANARY = -77


def _guarded(torch, a, shift=0):
    """A device copy of `a` between canary words, `shift` words off its 16-byte boundary; returns (view, check)."""
    a = np.ascontiguousarray(a)
    pad = np.full(16 + shift, CANARY & 0x7F, dtype=a.dtype)
    whole = torch.from_numpy(np.concatenate([pad, a.reshape(-1), pad])).cuda()
    view = whole[len(pad):len(pad) + a.size].view(a.shape)

    def check():
        h = whole.cpu().numpy()
        assert (h[:len(pad)] == pad).all() and (h[len(h) - len(pad):] == pad).all(), "written outside an array"
    return view, check


def _run(seq_lens, new_lens, width, *, free=None, spare=5, max_tokens=None, start=None, in_place=False, seed=0,
         tags=None, head=None, no_new=False, bad_ids=False, shift=0):
    torch = require_gpu()
    rng = np.random.default_rng(seed)
    lens, new = np.asarray(seq_lens, dtype=np.int32), np.asarray(new_lens, dtype=np.int32)
    b = len(lens)
    ok = (lens >= 0) & (new >= 0)
    need = int(np.where(ok, -(-(lens.astype(np.int64) + new) // 16) - -(-lens // 16), 0).clip(0, width).sum())
    count = need + spare if free is None else free
    cap = count + 3
    ids = rng.permutation(4 * cap + b * width).astype(np.int32)
    table = ids[cap:cap + b * width].reshape(b, width) if b else np.zeros((0, width), dtype=np.int32)
    ids = ids[:cap]
    num_blocks = 4 * cap + b * width
    if bad_ids:
        ids[::3] = num_blocks + 1 + np.arange(len(ids[::3]))
    tags = rng.integers(0, 2, size=(b, width)).astype(np.uint8) if tags is None else tags
    tail = np.minimum(np.maximum(lens, 0) // 16, width - 1)
    if tags is not None and b:
        tags[np.arange(b), tail] = tags[np.arange(b), tail] * 0 if tags.max() <= 1 else tags[np.arange(b), tail]
    head = cap - 2 if head is None else head
    rows = int(np.where(ok, new, 0).astype(np.int64).sum()) + 3 if max_tokens is None else max_tokens
    want = serve.extend(ids, head, count, num_blocks, lens, np.ones_like(new) if no_new else new, table, tags, rows, start)

    checks = []

    def dev(a, shift=0):
        v, c = _guarded(torch, a, shift)
        checks.append(c)
        return v

    d_ids, d_cur, d_lens, d_new = dev(ids), dev(np.array([head, count], dtype=np.int32)), dev(lens), dev(new)
    d_bt, d_tags = dev(table), dev(tags)
    d_cur_out = d_cur if in_place else dev(np.full(2, 9, dtype=np.int32))
    d_out = d_lens if in_place else dev(np.full(b, 9, dtype=np.int32))
    d_cu, d_slots, d_pos = (dev(np.full(n, 9, dtype=np.int32), k) for n, k in ((b + 1, 0), (rows, shift), (rows, shift)))
    d_status = dev(np.full(4, 9, dtype=np.int32))
    d_start = None if start is None else dev(np.asarray(start, dtype=np.int32))
    print(f"extend: B={b} rows={rows} need={need} free={count} in_place={in_place}", flush=True)
    ekv.extend(ekv.make_free_list(d_ids, d_cur, num_blocks, d_cur_out), d_lens, None if no_new else d_new, d_bt, d_tags,
               d_out, d_cu, d_slots, d_pos, d_status, d_start)
    torch.cuda.synchronize()
    for c in checks:
        c()
    got = dict(table=d_bt, tags=d_tags, lens=d_out, cu=d_cu, slots=d_slots, positions=d_pos, cursor=d_cur_out,
               status=d_status)
    for name, t in got.items():
        assert np.array_equal(t.cpu().numpy(), np.asarray(want[name])), (name, t.cpu().numpy(), want[name])
    if not in_place:
        assert np.array_equal(d_lens.cpu().numpy(), lens) and np.array_equal(d_cur.cpu().numpy(), [head, count])
    return want


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("case", [
    dict(seq_lens=[0], new_lens=[1], width=1), dict(seq_lens=[15], new_lens=[1], width=1),
    dict(seq_lens=[16], new_lens=[1], width=2), dict(seq_lens=[0], new_lens=[0], width=2),
    dict(seq_lens=[5, 16, 0, 31, 40], new_lens=[0, 16, 33, 1, 8], width=5),
    dict(seq_lens=[0, 0, 0], new_lens=[0, 0, 0], width=3), dict(seq_lens=[], new_lens=[], width=2)])
def test_small_tables(case, in_place):
    want = _run(**case, in_place=in_place)
    assert want["status"][0] == 0


@pytest.mark.parametrize("b", [63, 64, 65, 255, 257, 1000, 4096])
def test_decode_steps_of_many_sequences(b):
    rng = np.random.default_rng(b)
    lens = rng.integers(0, 300, size=b)
    assert _run(lens, np.ones(b), 20, seed=b, in_place=True)["status"][0] == 0
    assert _run(lens, np.ones(b), 20, seed=b, no_new=True, start=rng.integers(0, 9000, size=b))["status"][0] == 0


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("seed", range(3))
def test_ragged_prompts(seed, in_place):
    """Prompts from nothing to thousands of tokens beside decode steps, over several
    workgroups; a free list that lies across the end of its ring."""
    rng = np.random.default_rng(100 + seed)
    b = int(rng.integers(20, 300))
    lens = rng.integers(0, 700, size=b)
    new = np.where(rng.random(b) < 0.2, rng.integers(0, 4000, size=b), rng.integers(0, 2, size=b))
    assert _run(lens, new, 300, seed=seed, in_place=in_place, start=rng.integers(0, 100000, size=b))["status"][0] == 0


def test_one_very_long_prompt():
    assert _run([3, 0, 7], [1, 500001, 0], 31260, in_place=True)["status"][0] == 0


@pytest.mark.parametrize("shift", [0, 1])
@pytest.mark.parametrize("extra", [0, 1, 2, 3])
def test_more_tokens_than_threads(extra, shift):
    """Beyond 768 x 256 tokens a thread writes four neighbours: sequences of none, one
    and a few tokens between long ones, a last group that is not whole, rows behind the
    last token, and arrays that 16-byte stores would miss."""
    rng = np.random.default_rng(extra)
    new = np.concatenate([rng.integers(0, 4, size=500), [70001, 0, 0, 1, 130000], rng.integers(0, 40, size=60)])
    new[-1] += (extra - int(new.sum())) % 4
    lens = rng.integers(0, 90, size=len(new))
    want = _run(lens, new, 8200, seed=extra, shift=shift, start=rng.integers(0, 1000, size=len(new)))
    assert want["status"][0] == 0 and want["status"][1] > 768 * 256 and want["status"][1] % 4 == extra


@pytest.mark.parametrize("b", [256, 511, 769, 1024, 1025, 2049])
def test_numbers_of_sequences_around_a_wave_s_chunks(b):
    """A wave scans a quarter of the sequences, four chunks of 64 at a time."""
    rng = np.random.default_rng(b)
    assert _run(rng.integers(0, 200, size=b), rng.integers(0, 30, size=b), 20, seed=b)["status"][0] == 0


def test_a_refusal_among_many_sequences_takes_nothing():
    for at in (0, 63, 64, 600, 1026):
        new = np.full(1027, 2)
        new[at] = -1
        assert _run(np.full(1027, 7), new, 4, in_place=at % 2 == 0)["status"][0] == ekv.EXTEND_ROW


def test_exactly_all_free_blocks_and_rows():
    assert _run([0, 16], [32, 1], 4, spare=0, max_tokens=33)["status"] == (0, 33, 3, 0)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("case,reason", [
    (dict(seq_lens=[0, 60], new_lens=[3, 5], width=4), ekv.EXTEND_ROW), (dict(seq_lens=[-1, 0], new_lens=[1, 1], width=4), ekv.EXTEND_ROW),
    (dict(seq_lens=[1, 0], new_lens=[1, -1], width=4), ekv.EXTEND_ROW),
    (dict(seq_lens=[1, 0], new_lens=[2**31 - 1, 2**31 - 1], width=4, max_tokens=9), ekv.EXTEND_ROW),
    (dict(seq_lens=[0, 0], new_lens=[20, 20], width=4, max_tokens=39), ekv.EXTEND_TOKENS),
    (dict(seq_lens=[0, 0], new_lens=[20, 20], width=4, free=3), ekv.EXTEND_BLOCKS),
    (dict(seq_lens=[0, 0], new_lens=[20, 20], width=4, free=0, max_tokens=0), ekv.EXTEND_TOKENS | ekv.EXTEND_BLOCKS)])
def test_what_does_not_fit_takes_nothing(case, reason, in_place):
    assert _run(**case, in_place=in_place)["status"][0] == reason


def test_sums_beyond_32_bits_saturate():
    """4096 sequences of nearly 2^26 blocks each: the sums pass 2^31 many times over."""
    torch = require_gpu()
    b, width = 4096, (1 << 26) - 1
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    lens = torch.zeros(b, dtype=torch.int32, device="cuda")
    new = torch.full((b,), width * 16, dtype=torch.int32, device="cuda")
    out, cu = torch.empty_like(lens), torch.full((b + 1,), 9, dtype=torch.int32, device="cuda")
    slots, status, cursor = i32(5, 5, 5), i32(9, 9, 9, 9), i32(0, 4)
    ids, table = i32(1, 2, 3, 4), i32(0)   # (refused: no entry of the table is written; its lengths are 0, so none is read)
    ekv._check(ekv.lib().ekv_extend(ekv.FreeList(ids.data_ptr(), cursor.data_ptr(), cursor.data_ptr(), 4, 64), b, width,
                                    lens.data_ptr(), new.data_ptr(), None, table.data_ptr(), None, out.data_ptr(),
                                    cu.data_ptr(), 3, slots.data_ptr(), None, status.data_ptr(), None))
    torch.cuda.synchronize()
    assert status.tolist() == [ekv.EXTEND_TOKENS | ekv.EXTEND_BLOCKS, 1 << 30, 1 << 30, 4]
    assert not out.any() and not cu.any() and slots.tolist() == [-1, -1, -1] and cursor.tolist() == [0, 4]


def test_base_tail_is_refused():
    tags = np.zeros((3, 4), dtype=np.uint8)
    tags[1, 1] = 2   # (not reset by the helper: a partly filled block's tag)
    assert _run([16, 17, 0], [1, 1, 1], 4, tags=tags)["status"][0] == ekv.EXTEND_BASE
    tags[1, 1] = 0
    tags[:, 2:] = 1  # tags of blocks not in use yet say nothing
    assert _run([16, 17, 0], [1, 1, 1], 4, tags=tags)["status"][0] == 0


def test_ids_outside_the_pool_give_no_slot():
    want = _run([0, 5, 40], [70, 30, 90], 12, bad_ids=True)
    assert want["status"][0] == 0 and (want["slots"] == -1).sum() > 3


def test_cursor_outside_its_ring():
    assert _run([0, 5], [7, 30], 6, head=-1)["status"][0] == 0
    assert _run([0, 5], [7, 30], 6, head=1000)["status"][0] == 0


@pytest.mark.parametrize("steps", [40])
def test_paged_kv_grows_with_its_mirror(steps):
    """PagedKV.extend step by step, with demotions in between: device table, tags and
    lengths stay those of the mirror, and the free pool is used first in, first out."""
    torch = require_gpu()
    rng = np.random.default_rng(5)
    c = workloads.make_decode_case([40, 0, 129], 8, 2, seed=5, spare_blocks=90, max_blocks=40)
    kv = kvpool.PagedKV(c["pool"], c["block_table"], c["seq_lens"], c["free"], 2)
    start = torch.tensor([0, 1000, 7], dtype=torch.int32, device="cuda")
    for step in range(steps):
        before, free = kv.mirror.seq_lens.copy(), list(kv.mirror.free)
        new = rng.integers(0, 12 if step % 7 else 60, size=3) * (before < 500)
        if int((-(-(before + new) // 16) - -(-before // 16)).sum()) > len(free):
            with pytest.raises(ekv.EkvError):
                kv.extend(new)
            new = new * 0
        cu, slots, pos = kv.extend(new, start)
        assert np.array_equal(kv.bt.cpu().numpy(), kv.mirror.bt) and np.array_equal(kv.tags.cpu().numpy(), kv.mirror.tags)
        assert np.array_equal(kv.seq_lens.cpu().numpy(), kv.mirror.seq_lens)
        assert np.array_equal(cu.cpu().numpy(), np.concatenate([[0], np.cumsum(new)]))
        row = [(s, p) for s in range(3) for p in range(before[s], before[s] + new[s])]
        assert slots.tolist() == [int(kv.mirror.bt[s, p // 16]) * 16 + p % 16 for s, p in row]
        assert pos.tolist() == [p + int(start[s]) for s, p in row]
        assert list(kv.mirror.free) == free[len(free) - len(kv.mirror.free):]
        if step % 10 == 9:   # demote a full pair: its freed block goes to the back
            s = int(np.argmax(kv.mirror.seq_lens))
            j = next(j for j in range(20) if not kv.mirror.tags[s, 2 * j])
            kv.demote([[s, j]])
            kv.commit()


def test_extension_replays_from_a_graph():
    """A decode step's extension, in place, captured once: every replay continues
    from the state that the one before left, until the free list runs out."""
    torch = require_gpu()
    lens = np.array([3, 16, 0, 31], dtype=np.int32)
    table, tags = np.full((4, 6), -1, dtype=np.int32), np.zeros((4, 6), dtype=np.uint8)
    table[0, 0], table[1, 0], table[3, :2] = 90, 91, [92, 93]
    ids = np.arange(10, 17, dtype=np.int32)
    d = {k: torch.from_numpy(v).cuda() for k, v in dict(lens=lens, table=table, tags=tags, ids=ids).items()}
    cursor = torch.tensor([5, 6], dtype=torch.int32, device="cuda")
    cu, slots, pos, status = (torch.zeros(n, dtype=torch.int32, device="cuda") for n in (5, 6, 6, 4))
    free = ekv.make_free_list(d["ids"], cursor, 200)

    def step():
        ekv.extend(free, d["lens"], None, d["table"], d["tags"], d["lens"], cu, slots, pos, status)

    graph = torch.cuda.CUDAGraph()
    print("extend: capturing", flush=True)
    with torch.cuda.graph(graph):
        step()
    torch.cuda.synchronize()
    state = dict(lens=lens, table=table, tags=tags, cursor=(5, 6))
    refused = 0
    for replay in range(45):
        if replay % 5 == 4:
            step()   # eager work in between
        else:
            graph.replay()
        torch.cuda.synchronize()
        want = serve.extend(ids, *state["cursor"], 200, state["lens"], np.ones(4, dtype=np.int32), state["table"],
                            state["tags"], 6)
        for name, t in dict(table=d["table"], tags=d["tags"], lens=d["lens"], cu=cu, slots=slots, positions=pos,
                            cursor=cursor, status=status).items():
            assert np.array_equal(t.cpu().numpy(), np.asarray(want[name])), (replay, name)
        state = {k: want[k] for k in ("lens", "table", "tags", "cursor")}
        refused += want["status"][0] != 0
    assert refused > 0
