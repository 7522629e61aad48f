"""The long-context decode step on a cache whose pairs are demoted and refined between the
steps: bounds kept as it grows and refreshed from the first changed pair on, blocks of both
modes selected and attended, each step against the oracles of its operators on the words
that the GPU holds."""

import numpy as np
import pytest

from oracle import long_context as olc
from paper_2609_33536_amd import ekv, kvpool, workloads
from tests.context_util import expected_and_bound
from tests.gpu_util import default_scale, require_gpu

pytestmark = pytest.mark.gpu
HQ, HKV, BUDGET, SINK, RECENT = 8, 2, 9, 1, 2


@pytest.mark.parametrize("dtype", ["bf16", "e5m2"])
def test_a_decode_loop_with_transitions(dtype):
    torch = require_gpu()
    rng = np.random.default_rng(5)
    half = workloads.query_dtype(dtype)
    t = torch.bfloat16 if half == "bf16" else torch.float16
    c = workloads.make_decode_case([300, 33, 130], HQ, HKV, seed=5, base_fraction=0.0, dtype=dtype, spare_blocks=20, max_blocks=24)
    kv = kvpool.PagedKV(c["pool"], c["block_table"], c["seq_lens"], c["free"], HKV, dtype)
    b, elem = 3, c["pool"].dtype
    rope = ekv.make_rope(torch.from_numpy(ekv.rope_freqs(128, 10000.0).view(np.int64)).cuda(), 128)
    norm = ekv.make_head_norm(None, None, 1e-6)
    batch = kv.batch(HQ)
    bounds = ekv.key_bounds_buffer(kv.pool, batch)
    ekv.key_bounds(kv.pool, batch, bounds)
    ws_select, ws_decode = ekv.select_workspace(kv.pool, batch, BUDGET), ekv.decode_selected_workspace(kv.pool, batch, BUDGET)
    selected, counts = (torch.empty(x, dtype=torch.int32, device="cuda") for x in ((b, HKV, BUDGET), (b, HKV)))
    turned, out = torch.empty((b, HQ, 128), dtype=t, device="cuda"), torch.empty((b, HQ, 128), device="cuda")
    first, second = [[0, 2], [0, 5], [2, 0]], [[0, 0], [2, 2], [1, 0]]
    lo, attended = None, set()
    for step in range(12):
        known = kv.mirror.seq_lens.copy()   # (lengths before the new tokens, or the first changed pair's tokens)
        if step == 3:
            _, lo, _ = kv.demote(first)
        elif step == 6:
            kv.demote(second)
        elif step == 9:
            kv.refine(first, lo)
        for s, j in {3: first, 6: second, 9: first}.get(step, []):
            known[s] = min(known[s], 32 * j)
        kv.commit()
        _, slots, pos = kv.extend([1] * b)
        kv.relower()
        batch = kv.batch(HQ)
        q, k, v = (torch.from_numpy(rng.standard_normal((b, h, 128), dtype=np.float32) * 3).cuda().to(t) for h in (HQ, HKV, HKV))
        ekv.norm_rope_append(kv.pool, rope, norm, pos, slots, q, k, v, turned)
        ekv.key_bounds(kv.pool, batch, bounds, torch.from_numpy(known.astype(np.int32)).cuda())
        ekv.select_blocks(kv.pool, batch, turned, bounds, selected, counts, ws_select, SINK, RECENT)
        ekv.attn_decode_selected(kv.pool, batch, selected, counts, turned, out, default_scale(), ws_decode)
        torch.cuda.synchronize()
        lens, table, tags = kv.mirror.seq_lens, kv.mirror.bt, kv.mirror.tags
        assert lens.tolist() == [301 + step, 34 + step, 131 + step]
        assert np.array_equal(kv.bt.cpu().numpy(), table) and np.array_equal(kv.tags.cpu().numpy(), tags)
        pool = kv.kv.view(torch.uint8 if dtype == "e5m2" else torch.int16).cpu().numpy().view(elem).reshape(c["pool"].shape)
        got = bounds.cpu().numpy().view(elem)
        assert np.array_equal(got, olc.bounds(pool, table, tags, lens, [0] * b, got, dtype)), step
        qv = olc.values(turned.view(torch.int16).cpu().numpy().view(np.uint16), half)
        lists, n = selected.cpu().numpy(), counts.cpu().numpy()
        want, want_n = olc.select(qv, got, lens, BUDGET, SINK, RECENT, dtype)
        assert np.array_equal(n, want_n) and np.array_equal(lists, want), step
        result = out.cpu().numpy()
        for s in range(b):
            for h in range(HQ):
                mine = lists[s, h // 4, :n[s, h // 4]]
                attended |= {(step, int(tags[s, i])) for i in mine}
                x, y = olc.listed_tokens(pool, table[s], tags[s], lens[s], mine, h // 4, dtype)
                want, bound = expected_and_bound(qv[s, h], x, y, half, default_scale())
                assert (np.abs(result[s, h] - want) <= bound).all(), (step, s, h)
    assert {(4, 1), (7, 1), (11, 1), (11, 0)} <= attended   # BASE blocks among those that were attended
