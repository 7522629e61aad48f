"""The serving step's operators as they are used together: a decode loop over
sequences behind shared prefixes -- extension, rotary append, shared decode -- and
a prefill step, eager and from a captured graph, each step against the oracles of
its operators in turn."""

import numpy as np
import pytest

from oracle import attention as oatt
from oracle import encoding, serve
from paper_2609_33536_amd import ekv, workloads
from tests.gpu_util import check_attention, default_scale, require_gpu

pytestmark = pytest.mark.gpu
HQ, HKV, ROT, BASE = 8, 2, 128, 500000.0


def _dev(torch, a):
    a = np.ascontiguousarray(a)
    return torch.from_numpy(a.view(np.int16) if a.dtype == np.uint16 else a).cuda()


def _same_words(got, want):
    """Words of a rotation in 32 bits against one in 64, each rounded once: nearly all
    equal.  The two differ by at most 2^-20 (|x| + |y|) before the rounding, and where
    a rounding border lies between them by one step, eps = 2^-7 of the value, more.
    N(0, 1) words stay below 8, so that |x| + |y| <= 16 and the first part is at most
    2^-16: a turn that cancels (x cos near y sin) may leave a value far smaller than
    that, so a bound in steps of the result does not hold there."""
    a, b = encoding.words_to_f64(got, "bf16"), encoding.words_to_f64(want, "bf16")
    assert np.abs(b).max() < 8
    off = np.abs(a - b) - (2.0 ** -7 * np.abs(b) + 2.0 ** -16)
    assert off.max() <= 0, off.max()
    assert np.count_nonzero(got != want) <= 1e-3 * got.size


class _Oracle:
    """The step on the CPU: tables, lengths and pool words of its own."""

    def __init__(self, pool, table, lens, ids, head, count, theta):
        self.pool, self.table, self.lens, self.ids = pool.copy(), table.copy(), lens.copy(), ids
        self.tags, self.cursor, self.theta = np.zeros(table.shape, dtype=np.uint8), (head, count), theta

    def grow(self, new, start, rows):
        r = serve.extend(self.ids, *self.cursor, len(self.pool), self.lens, new, self.table, self.tags, rows, start)
        self.table, self.tags, self.lens, self.cursor = r["table"], r["tags"], r["lens"], r["cursor"]
        return r

    def store(self, slots, positions, q, k, v):
        """Rotates and appends; returns the queries as words."""
        turn = lambda w: workloads.f32_to_bf16_words(  # noqa: E731
            serve.rotate(encoding.words_to_f64(w, "bf16"), positions, self.theta, "half").astype(np.float32))
        live = slots >= 0
        blk, off = slots[live] // 16, slots[live] % 16
        self.pool[blk, 0, :, off] = turn(k)[live]
        self.pool[blk, 1, :, off] = v[live]
        return turn(q)


@pytest.mark.parametrize("graph", [False, True])
def test_decode_loop_behind_shared_prefixes(graph):
    """Two prefixes of 100 and 7 tokens, five sequences (one behind none), 40 steps:
    every step finds room, turns and stores the newest token and attends."""
    torch = require_gpu()
    rng = np.random.default_rng(1)
    prefix, start, own = np.array([100, 7], dtype=np.int32), [0, 3, 4], np.array([0, 15, 33, 16, 5], dtype=np.int32)
    b, nb, width = 5, 40, 6
    perm = rng.permutation(nb).astype(np.int32)
    pool = workloads.f32_to_bf16_words(rng.standard_normal((nb, 2, HKV, 16, 128), dtype=np.float32))
    ptable, at = np.zeros((2, 8), dtype=np.int32), 0
    table = np.zeros((b, width), dtype=np.int32)
    for t, lens in ((ptable, prefix), (table, own)):
        for s, n in enumerate(lens):
            t[s, :-(-n // 16)] = perm[at:at + -(-n // 16)]
            at += -(-n // 16)
    ids = perm[at:]
    behind = np.array([100, 100, 100, 7, 0], dtype=np.int32)   # each sequence's prefix tokens
    o = _Oracle(pool, table, own, ids, 3, len(ids), serve.frequencies(ROT, BASE))

    d_pool, d_table, d_lens, d_ids, d_ptable, d_prefix, d_behind = (
        _dev(torch, a) for a in (pool, table, own, ids, ptable, prefix, behind))
    cursor = torch.tensor([3, len(ids)], dtype=torch.int32, device="cuda")
    d_tags = torch.zeros((b, width), dtype=torch.uint8, device="cuda")
    empty = lambda *n: torch.empty(n, dtype=torch.int32, device="cuda")  # noqa: E731
    cu, slots, pos, status = empty(b + 1), empty(b), empty(b), empty(4)
    qkv = torch.empty((b, HQ + 2 * HKV, 128), dtype=torch.bfloat16, device="cuda")
    q, k, v = qkv[:, :HQ], qkv[:, HQ:HQ + HKV], qkv[:, HQ + HKV:]
    turned, out = torch.empty((b, HQ, 128), dtype=torch.bfloat16, device="cuda"), torch.empty((b, HQ, 128), device="cuda")
    kv = ekv.make_pool(d_pool, HKV)
    free = ekv.make_free_list(d_ids, cursor, nb)
    rope = ekv.make_rope(torch.from_numpy(ekv.rope_freqs(ROT, BASE).view(np.int64)).cuda(), ROT)
    prefixes = ekv.make_batch(d_prefix, d_ptable, None, None, HQ, ekv.MODE_NATIVE)
    batch = ekv.make_batch(d_lens, d_table, d_tags, None, HQ, ekv.MODE_NATIVE)
    starts = torch.tensor(start, dtype=torch.int32, device="cuda")
    ws = ekv.decode_shared_workspace(kv, prefixes, batch)

    def step():
        ekv.extend(free, d_lens, None, d_table, d_tags, d_lens, cu, slots, pos, status, d_behind)
        ekv.rope_append(kv, rope, pos, slots, q, k, v, turned)
        ekv.attn_decode_shared(kv, prefixes, starts, batch, turned, out, default_scale(), ws)

    run = step
    if graph:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step()
        run = g.replay
    for i in range(40):
        words = workloads.f32_to_bf16_words(rng.standard_normal((b, HQ + 2 * HKV, 128), dtype=np.float32))
        qkv.copy_(_dev(torch, words).view(torch.bfloat16))
        run()
        torch.cuda.synchronize()
        r = o.grow(np.ones(b, dtype=np.int32), behind, b)
        assert r["status"][0] == 0 and status.tolist() == list(r["status"])
        qw = o.store(r["slots"], r["positions"], words[:, :HQ], words[:, HQ:HQ + HKV], words[:, HQ + HKV:])
        for got, want in ((d_table, o.table), (d_lens, o.lens), (slots, r["slots"]), (pos, r["positions"]), (cursor, o.cursor)):
            assert np.array_equal(got.cpu().numpy(), np.asarray(want))
        _same_words(d_pool.cpu().numpy().view(np.uint16), o.pool)
        _same_words(turned.view(torch.int16).cpu().numpy().view(np.uint16), qw)
        # attention of the words that the GPU turned and stored (compared above)
        o.pool = d_pool.cpu().numpy().view(np.uint16).copy()
        qw = turned.view(torch.int16).cpu().numpy().view(np.uint16)
        want = serve.decode_shared(qw, o.pool, ptable, np.zeros_like(ptable, dtype=np.uint8), prefix, start, o.table, o.tags, o.lens)
        check_attention(out.cpu().numpy(), want, True)
    assert int(d_lens.sum()) == int(own.sum()) + 40 * b


def test_prefill_then_decode_step():
    """A chunk of ragged prompts: room by extension, rotary append of all its tokens
    into rows of a fixed number (the rest skipped), chunked prefill by the offsets
    that the extension made."""
    torch = require_gpu()
    rng = np.random.default_rng(2)
    own, new = np.array([20, 0, 64, 3], dtype=np.int32), np.array([30, 47, 1, 0], dtype=np.int32)
    b, nb, width, rows = 4, 40, 8, 100
    ids = rng.permutation(nb).astype(np.int32)
    table, at = np.zeros((b, width), dtype=np.int32), 0
    for s, n in enumerate(own):
        table[s, :-(-n // 16)] = ids[at:at + -(-n // 16)]
        at += -(-n // 16)
    ids = ids[at:]
    pool = workloads.f32_to_bf16_words(rng.standard_normal((nb, 2, HKV, 16, 128), dtype=np.float32))
    words = workloads.f32_to_bf16_words(rng.standard_normal((rows, HQ + 2 * HKV, 128), dtype=np.float32))
    o = _Oracle(pool, table, own, ids, 0, len(ids), serve.frequencies(ROT, BASE))
    r = o.grow(new, None, rows)
    qw = o.store(r["slots"], r["positions"], words[:, :HQ], words[:, HQ:HQ + HKV], words[:, HQ + HKV:])
    total = int(new.sum())
    d_pool, d_table, d_lens, d_ids, d_new = (_dev(torch, a) for a in (pool, table, own, ids, new))
    empty = lambda *n: torch.empty(n, dtype=torch.int32, device="cuda")  # noqa: E731
    cu, slots, pos, status = empty(b + 1), empty(rows), empty(rows), empty(4)
    cursor = torch.tensor([0, len(ids)], dtype=torch.int32, device="cuda")
    d_tags = torch.zeros((b, width), dtype=torch.uint8, device="cuda")
    qkv = _dev(torch, words).view(torch.bfloat16)
    kv = ekv.make_pool(d_pool, HKV)
    rope = ekv.make_rope(torch.from_numpy(ekv.rope_freqs(ROT, BASE).view(np.int64)).cuda(), ROT)
    turned = torch.empty((rows, HQ, 128), dtype=torch.bfloat16, device="cuda")
    out = torch.empty((rows, HQ, 128), device="cuda")
    ekv.extend(ekv.make_free_list(d_ids, cursor, nb), d_lens, d_new, d_table, d_tags, d_lens, cu, slots, pos, status)
    ekv.rope_append(kv, rope, pos, slots, qkv[:, :HQ], qkv[:, HQ:HQ + HKV], qkv[:, HQ + HKV:], turned)
    batch = ekv.make_batch(d_lens, d_table, d_tags, None, HQ, ekv.MODE_NATIVE)
    ekv.attn_prefill(kv, batch, turned, cu, int(new.max()), out, default_scale())
    torch.cuda.synchronize()
    assert np.array_equal(cu.cpu().numpy(), r["cu"]) and np.array_equal(d_table.cpu().numpy(), o.table)
    got_pool, got_q = d_pool.cpu().numpy().view(np.uint16), turned.view(torch.int16).cpu().numpy().view(np.uint16)
    _same_words(got_pool, o.pool)
    _same_words(got_q, qw)
    want = oatt.prefill(got_q[:total], r["cu"], got_pool, o.table, o.tags, o.lens)
    check_attention(out.cpu().numpy()[:total], want, True)
