"""Key bounds on the GPU against the oracle, word for word (nothing is rounded)."""

import numpy as np
import pytest

from oracle import long_context as olc
from paper_2609_33536_amd import ekv
from tests.context_util import Cache
from tests.gpu_util import require_gpu

pytestmark = pytest.mark.gpu


def _bounds(c, known, stream=None, old=None):
    torch = require_gpu()
    elem = c.pool.dtype
    shape = (len(c.lens), c.hkv, c.bt.shape[1], 2, 128)
    if old is None:
        old = np.random.default_rng(9).integers(0, np.iinfo(elem).max + 1, size=shape, dtype=elem)
    # (one row more: a canary)
    dev = torch.from_numpy(np.concatenate([old, old[:1]]).view(np.int16 if elem == np.uint16 else elem)).cuda()
    k = None if known is None else torch.tensor(np.asarray(known), dtype=torch.int32, device="cuda")
    ekv.key_bounds(c.kv.pool, c.batch, dev[:-1], k, stream)
    torch.cuda.synchronize()
    got = dev.cpu().numpy().view(elem)
    assert np.array_equal(got[-1], old[0])
    want = olc.bounds(c.pool, c.bt, c.tags, c.lens, [0] * len(c.lens) if known is None else known, old, c.dtype)
    assert np.array_equal(got[:-1], want)
    return dev


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "e5m2"])
@pytest.mark.parametrize("base", [0.0, 0.5, 1.0])
@pytest.mark.parametrize("structured", [True, False])
def test_types_fractions_and_modes(dtype, base, structured):
    print(f"bounds: {dtype} base={base} structured={structured}", flush=True)
    lens = [1, 15, 16, 17, 31, 32, 33, 64, 200, 0, 531]
    c = Cache(lens, 8, 2, dtype=dtype, base=base, structured=structured, seed=1)
    _bounds(c, None)
    _bounds(c, [0, 15, 0, 16, 30, 31, 32, 63, 77, 0, 300])
    _bounds(c, [max(0, n - 1) for n in lens])


@pytest.mark.parametrize("known", [0, 1, 15, 16, 17, 31, 32, 47, 48, 95, 96, 97, 1000, -5])
def test_known_tokens_around_blocks(known):
    c = Cache([96, 95, 97, 0, 30], 4, 4, seed=2, base=0.4, placement="oldest", max_blocks=12)
    _bounds(c, [max(0, known)] * 5) if known >= 0 else None
    torch = require_gpu()
    a, b = (ekv.key_bounds_buffer(c.kv.pool, c.batch) for _ in range(2))
    ekv.key_bounds(c.kv.pool, c.batch, a, torch.full((5,), known, dtype=torch.int32, device="cuda"))
    ekv.key_bounds(c.kv.pool, c.batch, b, torch.full((5,), max(0, known), dtype=torch.int32, device="cuda"))
    assert torch.equal(a, b)


@pytest.mark.parametrize("hkv,count", [(hkv, count) for hkv in (1, 3, 16) for count in (1, 63, 64, 65, 200)] + [(64, 1), (64, 20)])
def test_numbers_of_sequences_and_heads(hkv, count):
    """More sequences than a wave scans at once, and more units than waves."""
    rng = np.random.default_rng(count)
    lens = rng.integers(0, 90, size=count)
    lens[0] = 33
    c = Cache(lens, hkv, hkv, seed=hkv, base=0.3)
    _bounds(c, rng.integers(0, 60, size=count))


def test_more_units_than_waves():
    c = Cache([30001, 9000], 4, 4, dtype="e5m2", seed=4, base=0.5)
    _bounds(c, [0, 8500])
    _bounds(c, None)


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "e5m2"])
@pytest.mark.parametrize("base", [0.0, 1.0])
def test_all_bit_patterns(dtype, base):
    """Infinities, NaNs of both signs, subnormals and both zeros."""
    torch = require_gpu()
    rng = np.random.default_rng(6)
    c = Cache([160, 64], 4, 4, dtype=dtype, base=base, seed=6)
    elem = c.pool.dtype
    c.pool[:] = rng.integers(0, np.iinfo(elem).max + 1, size=c.pool.shape, dtype=elem)
    c.pool[:2] = 1 << (8 * elem.itemsize - 1)   # -0 beside 0
    c.pool[:2, :, :, ::3] = 0
    c.kv.kv.copy_(torch.from_numpy(c.pool.view(np.int16 if elem == np.uint16 else elem)).cuda().view(c.kv.kv.dtype).view(c.kv.kv.shape))
    _bounds(c, None)


def test_table_entries_outside_the_pool_and_stated_lengths():
    """Entries outside the pool are read as block 0, lengths up to the stated maximum."""
    torch = require_gpu()
    c = Cache([40, 70], 4, 2, seed=7)
    c.kv.bt[0, 1] = 10 ** 6
    c.kv.bt[1, 0] = -3
    c.bt = c.bt.copy()
    c.bt[0, 1] = c.bt[1, 0] = 0
    c.batch.max_seq_len = 50
    full = c.lens
    c.lens = np.minimum(full, 50)
    _bounds(c, None)
    assert torch.equal(c.kv.seq_lens.cpu(), torch.from_numpy(full))


def test_refresh_after_transitions():
    """Bounds of demoted pairs, and of refined ones, as the blocks are executed then."""
    torch = require_gpu()
    c = Cache([130, 64], 8, 2, seed=8, base=0.5, placement="oldest")
    base = _bounds(c, None).cpu()
    c2 = Cache([130, 64], 8, 2, seed=8, base=0.0, placement="oldest")
    target = _bounds(c2, None).cpu()
    changed = (base[:-1] != target[:-1]).flatten(3).any(-1)
    assert changed.any() and not changed[0, :, 8:].any()
    assert torch.equal(base[0, :, 8], target[0, :, 8])


def test_another_stream_and_a_graph():
    torch = require_gpu()
    c = Cache([100, 37], 8, 2, seed=9, max_blocks=12)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    _bounds(c, [3, 20], stream=side)
    lens, known = c.kv.seq_lens, torch.tensor([90, 30], dtype=torch.int32, device="cuda")
    c.batch.max_seq_len = 192
    out = ekv.key_bounds_buffer(c.kv.pool, c.batch)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ekv.key_bounds(c.kv.pool, c.batch, out, known)
    for replay in range(4):
        c.kv.kv.copy_(torch.randn(c.kv.kv.shape, device="cuda").bfloat16().view(torch.int16))
        lens.copy_(torch.tensor([100 - 20 * replay, 37 + replay], dtype=torch.int32))
        known.copy_(torch.tensor([40, 36], dtype=torch.int32))
        out.fill_(replay)
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        out.fill_(replay)
        ekv.key_bounds(c.kv.pool, c.batch, out, known)
        torch.cuda.synchronize()
        assert torch.equal(got, out)
