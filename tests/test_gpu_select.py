"""Block selection on the GPU against the oracle, whose scores are sums rounded once:
the lists have to be equal.  (Scores in 64 bits differ from those by less than 2^-45
of their size; random ones lie that close to each other with a chance of about
2^-40 a list.)"""

import numpy as np
import pytest

from oracle import long_context as olc
from paper_2609_33536_amd import ekv, workloads
from tests.gpu_util import require_gpu, words_to_tensor

pytestmark = pytest.mark.gpu


class Rows:
    """Bounds and queries of a batch, on both sides."""

    def __init__(self, lens, hq, hkv, dtype="bf16", seed=0, max_blocks=None, bounds=None, q=None):
        torch = require_gpu()
        rng = np.random.default_rng(seed)
        self.lens = np.asarray(lens, dtype=np.int32)
        b = len(self.lens)
        self.most = int(self.lens.max())
        width = max(2, -(-self.most // 16)) if max_blocks is None else max_blocks
        elem = np.uint8 if dtype == "e5m2" else np.uint16
        if bounds is None:
            x = rng.standard_normal((b, hkv, width, 2, 128), dtype=np.float32)
            bounds = workloads.to_words(np.sort(x * 2, axis=3), dtype)
            for s, length in enumerate(self.lens):   # rows behind the last block: anything
                n = -(-int(length) // 16)
                bounds[s, :, n:] = rng.integers(0, np.iinfo(elem).max + 1, size=bounds[s, :, n:].shape, dtype=elem)
        self.half = workloads.query_dtype(dtype)
        self.q = workloads.to_words(rng.standard_normal((b, hq, 128), dtype=np.float32), self.half) if q is None else q
        self.bounds, self.dtype, self.hkv = bounds, dtype, hkv
        self.d_bounds = torch.from_numpy(bounds.view(np.int16 if elem == np.uint16 else elem)).cuda()
        self.d_q = words_to_tensor(self.q, torch, self.half)
        self.d_lens = torch.from_numpy(self.lens).cuda()
        table = torch.zeros((b, width), dtype=torch.int32, device="cuda")
        self.kv = torch.zeros(2 * hkv * 2048, dtype=torch.uint8 if elem == np.uint8 else torch.int16, device="cuda")
        self.pool = ekv.make_pool(self.kv, hkv, dtype)
        self.table = table
        self.batch = ekv.make_batch(self.d_lens, table, None, None, hq, ekv.MODE_NATIVE, self.most)

    def select(self, budget, sink, recent, ws=None, stream=None):
        torch = require_gpu()
        b = len(self.lens)
        out = torch.full((b + 1, self.hkv, budget), 12345, dtype=torch.int32, device="cuda")
        counts = torch.full((b, self.hkv), -7, dtype=torch.int32, device="cuda")
        if ws is None:
            ws = ekv.select_workspace(self.pool, self.batch, budget)
            ws.fill_(0xFF)   # (nothing of it may matter)
        ekv.select_blocks(self.pool, self.batch, self.d_q, self.d_bounds, out[:b], counts, ws, sink, recent, stream)
        torch.cuda.synchronize()
        assert (out[b] == 12345).all()
        return out[:b].cpu().numpy(), counts.cpu().numpy()

    def check(self, budget, sink, recent, **kw):
        print(f"select: lens={len(self.lens)}x<={self.most} {self.dtype} Hq={self.q.shape[1]} Hkv={self.hkv} budget={budget} "
              f"sink={sink} recent={recent}", flush=True)
        got, counts = self.select(budget, sink, recent, **kw)
        want, want_counts = olc.select(olc.values(self.q, self.half), self.bounds, self.lens, budget, sink, recent, self.dtype)
        assert np.array_equal(counts, want_counts)
        assert np.array_equal(got, want), np.argwhere(got != want)[:4]


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "e5m2"])
@pytest.mark.parametrize("group", [1, 2, 4, 8, 16])
def test_types_and_groups(dtype, group):
    r = Rows([2000, 700, 1, 0, 16, 17, 1024, 1333], 2 * group, 2, dtype, seed=group)
    r.check(20, 1, 2)
    r.check(64, 0, 1)


@pytest.mark.parametrize("blocks", [1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 513, 1025])
def test_numbers_of_blocks(blocks):
    r = Rows([16 * blocks, 16 * blocks - 15], 4, 2, seed=blocks)
    for budget in (1, 2, 17, blocks, max(1, blocks - 1), blocks + 1):
        r.check(budget, 0, 0)


@pytest.mark.parametrize("sink,recent,budget", [(0, 0, 1), (1, 0, 1), (0, 1, 1), (1, 1, 2), (5, 3, 8), (5, 3, 9), (0, 12, 12),
                                                (12, 0, 13), (40, 40, 80), (30, 40, 100)])
def test_first_and_newest_blocks(sink, recent, budget):
    Rows([1600, 1590, 500, 79, 1285], 8, 2, seed=budget).check(budget, sink, recent)


@pytest.mark.parametrize("dtype", ["bf16", "e5m2"])
def test_long_rows(dtype):
    """More blocks than any part of the kernel takes at once."""
    r = Rows([200001, 70000], 4, 1, dtype, seed=3)
    r.check(256, 1, 4)
    r.check(2000, 0, 0)
    r.check(12000, 4, 4)


@pytest.mark.parametrize("sink,recent,budget", [(300, 0, 400), (0, 300, 400), (300, 299, 600), (300, 300, 600), (1, 2, 1199), (0, 0, 260)])
def test_first_and_newest_blocks_over_parts_of_a_row(sink, recent, budget):
    """Rows cut every few hundred blocks: parts that lie whole in the first or newest blocks, and shorter sequences."""
    Rows([1200 * 16, 1199 * 16 - 5, 700 * 16, 257 * 16, 0], 8, 2, seed=budget).check(budget, sink, recent)


def test_many_rows():
    rng = np.random.default_rng(4)
    Rows(rng.integers(0, 900, size=150), 8, 8, seed=4, max_blocks=70).check(16, 1, 1)


@pytest.mark.parametrize("budget", [1, 2, 40, 41, 99, 300, 599, 700])
@pytest.mark.parametrize("kinds", [1, 2, 7])
def test_equal_scores(budget, kinds):
    """Blocks of one, two and seven kinds: the lowest among equals."""
    rng = np.random.default_rng(kinds)
    x = workloads.to_words(np.sort(rng.standard_normal((kinds, 2, 128), dtype=np.float32), axis=1), "bf16")
    bounds = x[rng.integers(0, kinds, size=(2, 2, 600))]
    Rows([9600, 9000], 4, 2, bounds=bounds, seed=5).check(budget, 0, 1)


def test_neighbours_in_the_last_place():
    """Scores that differ by a 2^-30 of their size: 32 bits would call them equal."""
    n = 500
    v = np.zeros((1, 1, n, 2, 128), dtype=np.float32)
    v[..., 1, 0] = 2.0 ** 15
    v[0, 0, :, 1, 1] = np.random.default_rng(1).permutation(n) % 250 * 2.0 ** -7   # (fits 8 bits)
    q = workloads.to_words(np.ones((1, 1, 128), dtype=np.float32), "bf16")
    words = workloads.to_words(v, "bf16")
    assert np.array_equal(olc.values(words, "bf16"), v)
    Rows([16 * n], 1, 1, bounds=words, q=q).check(77, 0, 0)


def test_signs_and_zero_scores():
    """Negative scores, zeros of both signs (equal), and bounds of zero."""
    n = 300
    v = np.random.default_rng(2).integers(-3, 4, size=(1, 2, n, 1, 1)).astype(np.float32) * np.ones((1, 2, n, 2, 128), dtype=np.float32)
    v[:, :, ::5] = -0.0
    q = np.zeros((1, 2, 128), dtype=np.float32)
    q[0, 0, 3], q[0, 1, 4] = 1.0, -1.0
    r = Rows([16 * n], 2, 2, bounds=workloads.to_words(v, "bf16"), q=workloads.to_words(q, "bf16"))
    for budget in (10, 100, 150, 290):
        r.check(budget, 2, 3)


def test_infinite_and_undefined_scores():
    """A score that is no number is the largest, beside an infinite one."""
    n = 200
    v = np.sort(np.random.default_rng(3).standard_normal((1, 1, n, 2, 128)).astype(np.float32), axis=3)
    v[0, 0, 20, 1, 5] = np.inf
    v[0, 0, 21, 0, 6] = -np.inf
    v[0, 0, 100, 1, 7] = np.nan
    v[0, 0, 150, 0, 7] = np.nan
    q = np.random.default_rng(4).standard_normal((1, 2, 128)).astype(np.float32)
    q[0, :, 5], q[0, :, 6] = 1.0, [0.5, -0.5]
    words = workloads.to_words(v, "bf16")
    r = Rows([16 * n], 2, 1, bounds=words, q=workloads.to_words(q, "bf16"))
    got, _ = r.select(4, 0, 0)
    assert got[0, 0].tolist()[1:] == [21, 100, 150] or got[0, 0].tolist() == [20, 21, 100, 150]
    got, _ = r.select(2, 0, 0)
    assert got[0, 0].tolist() == [100, 150]


def test_workspace_shared_by_batches_and_a_stream():
    torch = require_gpu()
    big, small = Rows([3000, 2500], 8, 2, seed=6), Rows([500, 900, 30], 8, 2, seed=7)
    ws = ekv.select_workspace(big.pool, big.batch, 10)
    side = torch.cuda.Stream()
    for _ in range(2):
        big.check(10, 1, 1, ws=ws)
        small.check(10, 1, 1, ws=ws)
        side.wait_stream(torch.cuda.current_stream())
        big.check(10, 0, 0, ws=ws, stream=side)
        torch.cuda.current_stream().wait_stream(side)


@pytest.mark.parametrize("lens", [[3000, 40, 2000], [66000]])
def test_replayed_from_a_graph(lens):
    torch = require_gpu()
    r = Rows(lens, 8, 2, seed=8)
    ws = ekv.select_workspace(r.pool, r.batch, 24)
    out, counts = (torch.zeros(x, dtype=torch.int32, device="cuda") for x in ((len(lens), 2, 24), (len(lens), 2)))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ekv.select_blocks(r.pool, r.batch, r.d_q, r.d_bounds, out, counts, ws)
    for replay in range(4):
        r.d_q.copy_(torch.randn(r.d_q.shape, device="cuda"))
        r.d_lens.copy_(torch.tensor([max(1, n - 200 * replay) for n in lens], dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone(), counts.clone()
        out.fill_(9)
        ekv.select_blocks(r.pool, r.batch, r.d_q, r.d_bounds, out, counts, ws)
        torch.cuda.synchronize()
        assert torch.equal(got[0], out) and torch.equal(got[1], counts)
        r.q = r.d_q.view(torch.int16).cpu().numpy().view(np.uint16)
        r.lens = r.d_lens.cpu().numpy()
        r.check(24, 1, 1, ws=ws)
