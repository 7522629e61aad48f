"""Helpers of the long-context tests: seeded caches on both sides, and what the
arithmetic of decode over selected blocks may be off by."""

import math

import numpy as np

from oracle import fp8 as ofp8
from oracle import long_context as olc
from oracle import transitions as otr
from paper_2609_33536_amd import ekv, kvpool, workloads
from tests.attention_bound import U
from tests.gpu_util import host_safety_check, require_gpu, words_to_tensor


class Cache:
    """A cache on the GPU and the oracle's copy of it, some pairs BASE."""

    def __init__(self, lens, hq, hkv, *, dtype="bf16", base=0.0, placement="random", seed=0, structured=True, spare=3,
                 max_blocks=None):
        torch = require_gpu()
        c = workloads.make_decode_case(list(lens), hq, hkv, seed=seed, base_fraction=base, placement=placement, dtype=dtype,
                                       spare_blocks=spare, max_blocks=max_blocks)
        host_safety_check(c, c["pool"].shape)
        self.kv = kvpool.PagedKV(c["pool"], c["block_table"], c["seq_lens"], c["free"], hkv, dtype)
        self.pool, self.bt, self.tags, self.lens = c["pool"], c["block_table"], c["tags"], c["seq_lens"]
        if len(c["pairs"]):
            self.kv.demote(c["pairs"], emit_lo=False)
            self.pool, self.bt, self.tags, _, _ = (ofp8 if dtype == "e5m2" else otr).demote(
                self.pool, self.bt, self.tags, c["pairs"], self.lens)
        mode = self.kv.relower()
        if mode != ekv.MODE_NATIVE and not structured:
            mode = ekv.MODE_GENERAL
        self.batch = ekv.make_batch(self.kv.seq_lens, self.kv.bt, self.kv.tags, self.kv.bounds if structured else None, hq, mode,
                                    int(self.lens.max()))
        self.dtype, self.hq, self.hkv, self.q_words = dtype, hq, hkv, c["q"]
        self.half = workloads.query_dtype(dtype)
        self.q = words_to_tensor(c["q"], torch, self.half)
        self.q_values = olc.values(c["q"], self.half)


def expected_and_bound(q, k, v, dtype, scale):
    """Attention of one query [128] over k, v [n][128] in 64 bits, and the largest error
    of the kernel's arithmetic: the sums and roundings that tests/attention_bound.py
    counts, which are the same here (scores and their scale, powers of two, weights in two
    halves, sums in 32 bits, at most one change of reference a step of two blocks)."""
    if not len(k):
        return np.zeros(128), np.zeros(128)
    n = len(k)
    c = abs(scale) * math.log2(math.e)
    split, least = (2.0 ** -16, 0.0) if dtype == "bf16" else (2.0 ** -23, 2.0 ** -25)
    s, size = k @ q, np.abs(k) @ np.abs(q)
    t = math.copysign(c, scale) * s
    w = np.exp2(t - t.max())
    total = w.sum()
    e = math.log(2) * (c * 128 * 2 * U * size + 5 * U * np.abs(t) + U * np.abs(t).max()) + 2 * U
    out = w @ v / total
    units = -(-n // 16)   # (steps that are not full and pieces of the list: at most one a block)
    top = (w * (split + e + 4 * U * n + 8 * U * units) + least) @ np.abs(v) / total
    below = (w * (e + U * n + 8 * U * units)).sum() / total + 2 * U
    return out, 2 * (top + below * np.abs(out))
