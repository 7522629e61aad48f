"""Block selection where more scores are infinite or undefined than may be taken: the lists
against a sort of the scores (what is no number first, then the largest, the lowest block
first among equals), and no byte behind the lists or the workspace written."""

import numpy as np
import pytest

from oracle import long_context as olc
from paper_2609_33536_amd import ekv, workloads
from tests.gpu_util import require_gpu
from tests.test_gpu_select import Rows

pytestmark = pytest.mark.gpu
CANARY = 4096


def _rows(blocks, dtype, shares, sign, seed):
    """Rows of `blocks` blocks whose scores are NaN, +inf and -inf in the given shares, the others finite of one sign
    (1, -1) or both (0)."""
    rng = np.random.default_rng(seed)
    hkv, n = 2, max(blocks)
    v = np.zeros((len(blocks), hkv, n, 2, 128), dtype=np.float32)
    kind = rng.random(v.shape[:3])
    edges = np.cumsum(shares)
    size = rng.uniform(0.1, 9.0, size=v.shape[:3])
    v[..., 1, 0] = size * (sign if sign else rng.choice([-1.0, 1.0], size=v.shape[:3]))
    v[..., 1, 1] = np.where(kind < edges[0], np.nan, np.where(kind < edges[1], np.inf, np.where(kind < edges[2], -np.inf, 0.0)))
    q = np.zeros((len(blocks), 2 * hkv, 128), dtype=np.float32)
    q[..., :2] = 1.0
    return Rows([16 * b for b in blocks], 2 * hkv, hkv, dtype, bounds=workloads.to_words(v, dtype),
                q=workloads.to_words(q, workloads.query_dtype(dtype)))


def _ranked(r, budget, sink, recent):
    out = np.full((len(r.lens), r.hkv, budget), -1, dtype=np.int32)
    q = olc.values(r.q, r.half)
    for s, length in enumerate(r.lens):
        n = -(-int(length) // 16)
        for h in range(r.hkv):
            x = olc.values(r.bounds[s, h, :n], r.dtype)
            scores = olc.scores(q[s, 2 * h:2 * h + 2], x[:, 0], x[:, 1])
            middle = sorted(range(sink, n - recent), key=lambda i: (not np.isnan(scores[i]), -scores[i] if scores[i] == scores[i] else 0.0, i))
            chosen = [*range(sink), *range(n - recent, n), *middle[:budget - sink - recent]] if n > budget else [*range(n)]
            out[s, h, :len(chosen)] = sorted(chosen)
    return out


@pytest.mark.parametrize("blocks", [[300, 140, 301], [1200, 65, 700], [9000]])
@pytest.mark.parametrize("shares", [(0.8, 0.0, 0.0), (0.01, 0.0, 0.0), (0.0, 0.15, 0.0), (0.0, 0.7, 0.2), (0.2, 0.3, 0.3), (0.0, 0.0, 0.9),
                                    (1.0, 0.0, 0.0)])
@pytest.mark.parametrize("dtype,sign", [("bf16", 1), ("bf16", -1), ("bf16", 0), ("fp16", 0), ("e5m2", 0)])
def test_more_extreme_scores_than_are_taken(blocks, shares, dtype, sign):
    torch = require_gpu()
    r = _rows(blocks, dtype, shares, sign, seed=sum(blocks))
    for budget, sink, recent in ((1, 0, 0), (32, 0, 0), (40, 3, 5), (129, 1, 0)):
        print(f"extremes: {blocks} {dtype} {shares} sign={sign} budget={budget} sink={sink} recent={recent}", flush=True)
        size = ekv.select_workspace_bytes(r.pool, r.batch, budget)
        memory = torch.full((size + CANARY,), 0xA5, dtype=torch.uint8, device="cuda")
        got, counts = r.select(budget, sink, recent, ws=memory[:size])
        assert np.array_equal(got, _ranked(r, budget, sink, recent))
        assert (counts == np.minimum(-(-r.lens // 16), budget)[:, None]).all()
        assert bool((memory[size:] == 0xA5).all())


@pytest.mark.parametrize("budget,want", [(1, [100]), (2, [100, 150]), (3, [20, 100, 150]), (4, [20, 21, 100, 150])])
def test_what_is_no_number_comes_before_infinity_and_that_by_block(budget, want):
    n = 200
    v = np.sort(np.random.default_rng(3).standard_normal((1, 1, n, 2, 128)).astype(np.float32), axis=3)
    v[0, 0, 20, 1, 5], v[0, 0, 21, 0, 6], v[0, 0, 100, 1, 7], v[0, 0, 150, 0, 7] = np.inf, -np.inf, np.nan, np.nan
    q = np.random.default_rng(4).standard_normal((1, 2, 128)).astype(np.float32)
    q[0, :, 5], q[0, :, 6] = 1.0, [0.5, -0.5]
    r = Rows([16 * n], 2, 1, bounds=workloads.to_words(v, "bf16"), q=workloads.to_words(q, "bf16"))
    assert r.select(budget, 0, 0)[0][0, 0].tolist() == want


@pytest.mark.parametrize("lens", [[2000, 700, 333], [19200, 700, 16000]])
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "e5m2"])
@pytest.mark.parametrize("group,head,sign", [(1, 0, 0), (4, 3, 1), (16, 9, 0)])
def test_queries_that_are_no_numbers(lens, dtype, group, head, sign):
    """Every score of their KV head is undefined then: the first blocks among equals.  Other heads and sequences keep
    their lists."""
    half = workloads.query_dtype(dtype)
    q = workloads.to_words(np.random.default_rng(group).standard_normal((3, 2 * group, 128), dtype=np.float32), half)
    q[1, head, 77] = (0x7FC0 if half == "bf16" else 0x7E00) | sign << 15
    r = Rows(lens, 2 * group, 2, dtype, seed=group, q=q)
    r.check(20, 1, 2)
    r.check(30, 0, 0)
    got, _ = r.select(20, 1, 2)
    n = -(-lens[1] // 16)
    assert got[1, 0].tolist() == [*range(18), n - 2, n - 1]
