"""Decode over selected blocks on the GPU against the oracle in 64 bits, within the
bound of its arithmetic (tests/context_util.py); 16-bit outputs add their rounding,
half a step."""

import numpy as np
import pytest

from oracle import long_context as olc
from paper_2609_33536_amd import ekv, workloads
from tests.context_util import Cache, expected_and_bound
from tests.gpu_util import default_scale, require_gpu, words_to_tensor

pytestmark = pytest.mark.gpu


def _lists(c, budget, seed=0, order="ascending", counts=None, strays=False):
    """A list for every (sequence, KV head): random blocks of the sequence, at most the budget."""
    rng = np.random.default_rng(seed)
    selected = np.full((len(c.lens), c.hkv, budget), -1, dtype=np.int32)
    n_out = np.zeros((len(c.lens), c.hkv), dtype=np.int32)
    for s, length in enumerate(c.lens):
        n = -(-int(length) // 16)
        for h in range(c.hkv):
            take = min(n, budget) if counts is None else min(n, budget, int(rng.integers(0, budget + 1)))
            pick = rng.permutation(n)[:take]
            if take and rng.random() < 0.7 and n - 1 not in pick:
                pick[0] = n - 1   # the block that the sequence ends in
            pick = np.sort(pick) if order == "ascending" else pick
            if strays:   # entries that are no blocks, anywhere
                pick = np.concatenate([pick, rng.choice([-1, n, n + 7, 10 ** 9, -2 ** 31], size=budget)])[:budget]
                pick = rng.permutation(pick)
            selected[s, h, :len(pick)] = pick
            n_out[s, h] = len(pick)
    return selected, n_out


def _check(c, selected, counts, out, scale):
    dtype = "fp16" if out.dtype == np.float16 else ("fp32" if out.dtype == np.float32 else "bf16")
    half = {"fp32": 0.0, "bf16": 2.0 ** -8, "fp16": 2.0 ** -11}[dtype]
    group = c.hq // c.hkv
    got = out.astype(np.float64) if dtype != "bf16" else olc.values(out, "bf16")
    worst = 0.0
    for s in range(len(c.lens)):
        for h in range(c.hkv):
            k, v = olc.listed_tokens(c.pool, c.bt[s], c.tags[s], c.lens[s], selected[s, h, :counts[s, h]], h, c.dtype)
            for g in range(h * group, (h + 1) * group):
                want, bound = expected_and_bound(c.q_values[s, g], k, v, c.half, scale)
                bound = bound + half * (np.abs(want) + bound) + (2.0 ** -25 if dtype == "fp16" else 0.0)
                off = np.abs(got[s, g] - want)
                bad = ~(off <= bound)
                assert not bad.any(), (s, h, g, int(bad.argmax()), got[s, g][bad][0], want[bad][0], bound[bad][0])
                worst = max(worst, float(np.max(off / np.maximum(bound, 1e-300))))
    print(f"worst {worst:.3f} of the bound", flush=True)


def _decode(c, selected, counts, *, fp32=True, scale=None, ws=None, stream=None, pass_counts=True):
    torch = require_gpu()
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()  # noqa: E731
    out = torch.full(c.q.shape, float("nan"), dtype=torch.float32 if fp32 else c.q.dtype, device="cuda")
    ws = ekv.decode_selected_workspace(c.kv.pool, c.batch, selected.shape[2]) if ws is None else ws
    ekv.attn_decode_selected(c.kv.pool, c.batch, dev(selected), dev(counts) if pass_counts else None, c.q, out,
                             default_scale() if scale is None else scale, ws, stream)
    torch.cuda.synchronize()
    if fp32:
        return out.cpu().numpy()
    return out.cpu().numpy() if out.dtype == torch.float16 else out.view(torch.int16).cpu().numpy().view(np.uint16)


def _run(lens, hq, hkv, budget, *, fp32=True, scale=None, seed=0, order="ascending", ragged=None, strays=False, pass_counts=True, **kw):
    print(f"selected: B={len(lens)} Hq={hq} Hkv={hkv} budget={budget} fp32={fp32} {order} {kw}", flush=True)
    c = Cache(lens, hq, hkv, seed=seed, **kw)
    selected, counts = _lists(c, budget, seed, order, ragged, strays)
    if not pass_counts:
        counts = np.full_like(counts, budget)
    out = _decode(c, selected, counts, fp32=fp32, scale=scale, pass_counts=pass_counts)
    _check(c, selected, counts, out, default_scale() if scale is None else scale)


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "e5m2"])
@pytest.mark.parametrize("base", [0.0, 0.5, 1.0])
@pytest.mark.parametrize("group", [1, 2, 4, 8, 16])
def test_groups_types_and_fractions(dtype, base, group):
    _run([700, 33, 1, 0, 16, 490], 2 * group, 2, 21, dtype=dtype, base=base, seed=group)


@pytest.mark.parametrize("fp32", [True, False])
@pytest.mark.parametrize("structured", [True, False])
@pytest.mark.parametrize("dtype", ["bf16", "e5m2", "fp16"])
def test_oldest_half_base_structured_and_general(fp32, structured, dtype):
    _run([900, 1024, 511], 16, 4, 30, dtype=dtype, base=0.5, placement="oldest", structured=structured, fp32=fp32, seed=3)


@pytest.mark.parametrize("budget", [1, 2, 3, 4, 7, 8, 9, 15, 16, 17, 31, 33, 63, 64, 65, 130])
def test_budgets(budget):
    """Odd and even lists, fewer steps than waves, one and several workgroups a list."""
    _run([2100, 40, 1111], 8, 2, budget, seed=budget, base=0.3)


@pytest.mark.parametrize("length", [1, 2, 15, 16, 17, 31, 32, 33, 47, 48, 49, 64, 65])
@pytest.mark.parametrize("dtype", ["bf16", "e5m2"])
def test_lengths_around_blocks(length, dtype):
    _run([length] * 3, 8, 2, 8, seed=length, dtype=dtype)


@pytest.mark.parametrize("dtype", ["bf16", "e5m2"])
@pytest.mark.parametrize("order", ["ascending", "any"])
def test_ragged_lists_in_any_order_with_strays(dtype, order):
    _run([800, 0, 5, 333, 64], 8, 4, 19, dtype=dtype, base=0.4, order=order, ragged=True, seed=11)
    _run([800, 0, 5, 333, 64], 8, 4, 19, dtype=dtype, base=0.4, order=order, ragged=True, strays=True, seed=12)
    _run([800, 0, 5, 333, 64], 8, 4, 19, dtype=dtype, base=0.4, strays=True, pass_counts=False, seed=13)


def test_counts_outside_the_budget_are_clamped():
    c = Cache([300, 300], 4, 2, seed=14)
    selected, counts = _lists(c, 6)
    a = _decode(c, selected, np.array([[6, 0], [6, 6]]))
    b = _decode(c, selected, np.array([[10 ** 6, -5], [7, 2 ** 31 - 1]]))
    assert np.array_equal(a, b) and (a[0, 2:] == 0).all()


@pytest.mark.parametrize("scale", [-0.3, 0.0, -0.0, 1.0, 0.01])
@pytest.mark.parametrize("dtype", ["bf16", "e5m2"])
def test_softmax_scales(scale, dtype):
    _run([400, 70], 8, 2, 12, scale=scale, dtype=dtype, base=0.5, seed=31)


def _repeated(batch, blocks, hq, hkv, dtype, seed=0, length=None):
    """Many long sequences over one small pool: every table row is a permutation of it."""
    torch = require_gpu()
    c = Cache([16 * blocks], hq, hkv, dtype=dtype, seed=seed, spare=0, max_blocks=blocks)
    rng = np.random.default_rng(seed)
    c.bt = np.stack([rng.permutation(blocks) for _ in range(batch)]).astype(np.int32)
    c.tags = np.zeros_like(c.bt, dtype=np.uint8)
    c.lens = np.full(batch, 16 * blocks - 3 if length is None else length, dtype=np.int32)
    c.q_words = workloads.to_words(rng.standard_normal((batch, hq, 128), dtype=np.float32), c.half)
    c.q, c.q_values = words_to_tensor(c.q_words, torch, c.half), olc.values(c.q_words, c.half)
    c.device = [torch.from_numpy(x).cuda() for x in (c.lens, c.bt)]
    c.batch = ekv.make_batch(*c.device, None, None, hq, ekv.MODE_NATIVE, int(c.lens[0]))
    return c


@pytest.mark.parametrize("dtype", ["bf16", "e5m2"])
@pytest.mark.parametrize("budget", [255, 256, 257, 300, 391])
def test_lists_of_several_windows(dtype, budget):
    """70 x 8 lists, each in one workgroup: more than 64 entries a wave."""
    c = _repeated(70, 400, 8, 8, dtype, seed=budget)
    selected, counts = _lists(c, budget, budget)
    _check(c, selected, counts, _decode(c, selected, counts), default_scale())


@pytest.mark.parametrize("batch,hkv,budget", [(1, 1, 1000), (1, 8, 512), (3, 4, 200), (63, 8, 40), (64, 8, 40), (65, 8, 40),
                                              (16, 8, 200), (32, 8, 130), (33, 8, 130), (48, 8, 129), (49, 8, 128)])
def test_workgroups_to_a_list(batch, hkv, budget):
    c = _repeated(batch, 1024 if budget > 600 else 520, 2 * hkv, hkv, "bf16", seed=budget)
    selected, counts = _lists(c, budget, 1)
    _check(c, selected, counts, _decode(c, selected, counts), default_scale())


@pytest.mark.parametrize("lengths", [[1, 2, 3], [40, 17, 0], [500, 512, 1]])
@pytest.mark.parametrize("batch,budget", [(1, 700), (13, 165), (3, 33)])
def test_budgets_beyond_the_sequences(lengths, batch, budget):
    """Fewer blocks than the budget has room for, with strays behind them: workgroups go by the blocks."""
    c = Cache(lengths * batch, 16, 8, seed=budget)
    n = -(-max(lengths) // 16)
    selected = np.full((3 * batch, 8, budget), -1, dtype=np.int32)
    selected[:, :, :n] = np.arange(n)
    counts = np.full((3 * batch, 8), budget)
    _check(c, selected, counts, _decode(c, selected, counts), default_scale())


def test_all_blocks_are_the_dense_decode():
    torch = require_gpu()
    c = Cache([500, 77, 0, 1029], 32, 8, base=0.4, seed=16)
    n = c.bt.shape[1]
    selected = np.broadcast_to(np.arange(n, dtype=np.int32), (4, 8, n)).copy()
    out = _decode(c, selected, np.full((4, 8), n))
    dense = torch.empty_like(c.q, dtype=torch.float32)
    ekv.attn_decode(c.kv.pool, c.batch, c.q, dense, default_scale(), ekv.decode_workspace(c.kv.pool, c.batch))
    torch.cuda.synchronize()
    assert np.abs(out - dense.cpu().numpy()).max() <= 2e-5   # (both within their bound, some 1e-5 for unit values)
    _check(c, selected, np.full((4, 8), n), out, default_scale())


def test_bad_values_in_blocks_that_are_not_listed():
    torch = require_gpu()
    c = Cache([640], 8, 2, seed=17)
    selected = np.array([[[1, 5, 30, 39]] * 2], dtype=np.int32)
    want = _decode(c, selected, np.full((1, 2), 4))
    for i in range(40):
        if i not in (1, 5, 30, 39):
            c.kv.kv.view(torch.int16).view(-1, 2 * 2 * 2048)[int(c.bt[0, i])] = 0x7FC0   # NaN
    assert np.array_equal(_decode(c, selected, np.full((1, 2), 4)), want)


@pytest.mark.parametrize("first", [True, False])
def test_scores_of_minus_infinity_weigh_nothing(first):
    """Keys with -inf where the query is positive: the softmax leaves them out, also where a wave meets nothing else."""
    torch = require_gpu()
    c = Cache([160], 2, 1, seed=18)
    c.q_words[0, :, 0] = 0x3F80   # 1.0
    c.q, c.q_values = words_to_tensor(c.q_words, torch, "bf16"), olc.values(c.q_words, "bf16")
    gone = [0, 1, 2] if first else [7, 8, 4]
    for i in gone:
        c.pool[c.bt[0, i], 0, 0, :, 0] = 0xFF80
    c.kv.kv.copy_(torch.from_numpy(c.pool.view(np.int16)).cuda().view(c.kv.kv.dtype).view(c.kv.kv.shape))
    every = np.arange(10, dtype=np.int32).reshape(1, 1, 10)
    out = _decode(c, every, np.full((1, 1), 10))
    rest = np.array([[[i for i in range(10) if i not in gone]]], dtype=np.int32)
    _check(c, rest, np.full((1, 1), 7), out, default_scale())


def test_a_pool_beyond_32_bits():
    """Blocks whose bytes begin beyond 4 GiB."""
    torch = require_gpu()
    c = Cache([200, 90], 8, 8, seed=19)
    far, n = 70000, len(c.pool)
    kv = torch.zeros((far + n, 2, 8, 16, 128), dtype=torch.int16, device="cuda")
    kv[far:] = torch.from_numpy(c.pool.view(np.int16)).cuda()
    c.kv.bt += far
    selected, counts = _lists(c, 9)
    c.kv.pool = ekv.make_pool(kv, 8)
    _check(c, selected, counts, _decode(c, selected, counts), default_scale())


def test_workspace_shared_by_batches_streams_and_repeats():
    torch = require_gpu()
    a, b = Cache([900, 300], 8, 2, seed=20), Cache([50, 1400, 700], 16, 4, seed=21, base=0.5)
    lists = {id(x): _lists(x, 40, 5) for x in (a, b)}
    ws = torch.zeros(max(ekv.decode_selected_workspace_bytes(x.kv.pool, x.batch, 40) for x in (a, b)), dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    first = {}
    for turn in range(3):
        for x in (a, b):
            out = _decode(x, *lists[id(x)], ws=ws)
            _check(x, *lists[id(x)], out, default_scale())
            assert np.array_equal(first.setdefault(id(x), out), out)   # the same sums every time
        side.wait_stream(torch.cuda.current_stream())
        assert np.array_equal(_decode(a, *lists[id(a)], ws=ws, stream=side), first[id(a)])
    assert not ws[:32768].any()   # the counters are back at zero


def test_workspace_shared_with_the_dense_decode():
    """In turn on one workspace, both with lists and sequences that are cut."""
    torch = require_gpu()
    c = Cache([4000, 900], 32, 8, seed=23, base=0.3)
    n = c.bt.shape[1]
    selected = np.broadcast_to(np.arange(n, dtype=np.int32), (2, 8, n)).copy()
    sizes = ekv.decode_selected_workspace_bytes(c.kv.pool, c.batch, n), ekv.decode_workspace(c.kv.pool, c.batch).numel()
    ws = torch.zeros(max(sizes), dtype=torch.uint8, device="cuda")
    dense = torch.empty_like(c.q, dtype=torch.float32)
    for _ in range(3):
        out = _decode(c, selected, np.full((2, 8), n), ws=ws)
        dense.fill_(7)
        ekv.attn_decode(c.kv.pool, c.batch, c.q, dense, default_scale(), ws)
        torch.cuda.synchronize()
        _check(c, selected, np.full((2, 8), n), out, default_scale())
        assert np.abs(out - dense.cpu().numpy()).max() <= 2e-5   # (as test_all_blocks_are_the_dense_decode)


@pytest.mark.parametrize("batch", [2, 70])
def test_replayed_from_a_graph(batch):
    torch = require_gpu()
    c = _repeated(batch, 200, 32, 8, "bf16", seed=22)
    budget = 50
    ws = ekv.decode_selected_workspace(c.kv.pool, c.batch, budget)
    sel, cnt = (torch.zeros(x, dtype=torch.int32, device="cuda") for x in ((batch, 8, budget), (batch, 8)))
    out = torch.empty_like(c.q)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ekv.attn_decode_selected(c.kv.pool, c.batch, sel, cnt, c.q, out, default_scale(), ws)
    for replay in range(4):
        selected, counts = _lists(c, budget, replay, counts=True)
        sel.copy_(torch.from_numpy(selected)), cnt.copy_(torch.from_numpy(counts))
        c.q.copy_(torch.randn(c.q.shape, device="cuda"))
        out.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        ekv.attn_decode_selected(c.kv.pool, c.batch, sel, cnt, c.q, out, default_scale(), ws)
        torch.cuda.synchronize()
        assert torch.equal(got, out)
    c.q_values = olc.values(c.q.view(torch.int16).cpu().numpy().view(np.uint16), "bf16")
    _check(c, selected, counts, got.view(torch.int16).cpu().numpy().view(np.uint16), default_scale())
