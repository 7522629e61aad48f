"""The long-context oracle against other ways to say the same."""

import numpy as np
import pytest

from oracle import attention, long_context as olc
from oracle import fp8 as ofp8
from oracle import transitions as otr
from paper_2609_33536_amd import workloads


def _case(dtype, base=0.5, seed=0, lens=(70, 1, 0, 33, 129), hq=8, hkv=2):
    c = workloads.make_decode_case(list(lens), hq, hkv, seed=seed, base_fraction=base, dtype=dtype, garbage_tail=False)
    pool, bt, tags = c["pool"], c["block_table"], c["tags"]
    if len(c["pairs"]):
        pool, bt, tags, _, _ = (ofp8 if dtype == "e5m2" else otr).demote(pool, bt, tags, c["pairs"], c["seq_lens"])
    half = workloads.query_dtype(dtype)
    return c, pool, bt, tags, olc.values(c["q"], half)


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "e5m2"])
def test_bounds_are_the_extreme_values(dtype):
    c, pool, bt, tags, _ = _case(dtype)
    old = np.full((5, 2, bt.shape[1], 2, 128), 77, dtype=pool.dtype)
    known = [32, 0, 0, 40, 16]
    got = olc.bounds(pool, bt, tags, c["seq_lens"], known, old, dtype)
    for s, length in enumerate(c["seq_lens"]):
        for i in range(bt.shape[1]):
            if known[s] // 16 <= i < -(-int(length) // 16):
                x = olc.values(olc.block_keys(pool, bt[s], tags[s], i, dtype), dtype)[:, :int(length) - 16 * i]
                assert np.array_equal(olc.values(got[s, :, i, 0], dtype), x.min(axis=1))
                assert np.array_equal(olc.values(got[s, :, i, 1], dtype), x.max(axis=1))
            else:
                assert (got[s, :, i] == 77).all()


def test_order_of_words():
    words = np.array([0xFFFF, 0xFF80, 0xC000, 0x8001, 0x8000, 0, 1, 0x4000, 0x7F80, 0x7FFF], dtype=np.uint16)
    assert (np.diff(olc._order(words)) > 0).all()
    assert (np.diff(olc._order(np.array([0xFF, 0xFC, 0x81, 0x80, 0, 1, 0x7C, 0x7F], dtype=np.uint8))) > 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "e5m2"])
def test_scores_bound_every_key(dtype):
    c, pool, bt, tags, q = _case(dtype)
    b = olc.bounds(pool, bt, tags, c["seq_lens"], [0] * 5, np.zeros((5, 2, bt.shape[1], 2, 128), dtype=pool.dtype), dtype)
    for s, length in enumerate(c["seq_lens"]):
        for h in range(2):
            n = -(-int(length) // 16)
            x = olc.values(b[s, h, :n], dtype)
            top = olc.scores(q[s, 4 * h:4 * h + 4], x[:, 0], x[:, 1])
            for i in range(n):
                k, _ = olc.listed_tokens(pool, bt[s], tags[s], length, [i], h, dtype)
                assert (k @ q[s, 4 * h:4 * h + 4].sum(axis=0) <= top[i] + 1e-9).all()


def test_select_takes_the_largest_and_the_first_among_equals():
    b = np.zeros((1, 1, 6, 2, 128), dtype=np.uint16)
    b[0, 0, :, 1, 0] = [0, 0x3F80, 0x4000, 0x3F80, 0x3F80, 0]   # 0 1 2 1 1 0
    q = np.zeros((1, 1, 128))
    q[..., 0] = 1.0
    pick = lambda *a: olc.select(q, b, [96], *a, "bf16")[0][0, 0].tolist()  # noqa: E731
    assert pick(1, 0, 0) == [2] and pick(3, 0, 0) == [1, 2, 3] and pick(3, 1, 1) == [0, 2, 5]
    assert pick(4, 0, 2) == [1, 2, 4, 5] and pick(7, 1, 1) == [0, 1, 2, 3, 4, 5, -1]


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_decode_of_all_blocks_is_the_dense_decode(dtype):
    c, pool, bt, tags, q = _case(dtype)
    n = bt.shape[1]
    rng = np.random.default_rng(3)
    every = np.array([[rng.permutation(n + 2) - 1 for _ in range(2)] for _ in range(5)])   # -1 and n: no blocks
    got = olc.decode(q, pool, bt, tags, c["seq_lens"], every, np.full((5, 2), n + 2), dtype)
    want = attention.decode(c["q"], pool, bt, tags, c["seq_lens"], dtype)
    assert np.abs(got - want).max() < 1e-12


def test_level_makes_the_mean_square_one():
    x = np.random.default_rng(1).standard_normal((4, 3, 128)) * 7
    y = olc.level(x, None, 1e-12)
    assert np.allclose((y * y).mean(axis=-1), 1.0)
    w = np.random.default_rng(2).standard_normal((3, 128))
    assert np.allclose(olc.level(x, w, 1e-12, 1.0), y * (w + 1.0))
    assert (olc.level(np.zeros((1, 1, 128)), w[:1], 1e-6) == 0).all()
