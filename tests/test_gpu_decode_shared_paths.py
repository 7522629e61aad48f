"""Shared-prefix decode where short batches do not reach (the host check of the same
cases proves that they do), and to the last bits that its arithmetic keeps."""

import numpy as np
import pytest

from oracle import encoding, serve
from oracle import fp8 as ofp8
from oracle import transitions as otr
from paper_2609_33536_amd import ekv, kvpool, workloads
from tests.attention_bound import expected_and_bound
from tests.gpu_util import default_scale, host_safety_check, require_gpu, words_to_tensor
from tests.shared_plan.cases import CASES

pytestmark = pytest.mark.gpu


class Batch:
    """Prefixes and sequences in one table, their pairs demoted as asked, on both sides."""

    def __init__(self, prefix, own, start, hq, hkv, dtype="bf16", base=0.0, base_of="both", seed=0, positive=False, whole=False,
                 placement="random"):
        torch = require_gpu()
        n, self.hq, self.hkv, self.dtype, self.own, self.prefix = len(prefix), hq, hkv, dtype, list(own), list(prefix)
        c = workloads.make_decode_case(self.prefix + self.own, hq, hkv, seed=seed, base_fraction=base, placement=placement,
                                       dtype=dtype, spare_blocks=3)
        host_safety_check(c, c["pool"].shape)
        pool = c["pool"].copy()
        if whole:      # values that 32 bits sum exactly
            x = np.random.default_rng(seed + 1).integers(-2, 3, size=pool[:, 1].shape).astype(np.float32)
            pool[:, 1] = workloads.to_words(x, dtype).reshape(x.shape)
        if positive:   # values of one sign: what a weight loses does not average out
            pool[:, 1] &= 0x7F if dtype == "e5m2" else 0x7FFF
        pairs = np.asarray(c["pairs"], dtype=np.int32).reshape(-1, 2)
        pairs = pairs[{"both": slice(None), "prefix": pairs[:, 0] < n, "own": pairs[:, 0] >= n}[base_of]]
        self.kv = kvpool.PagedKV(pool, c["block_table"], c["seq_lens"], c["free"], hkv, dtype)
        self.pool, self.table, self.tags = pool, c["block_table"], c["tags"]
        if len(pairs):
            self.kv.demote(pairs, emit_lo=False)
            self.pool, self.table, self.tags, _, _ = (ofp8 if dtype == "e5m2" else otr).demote(pool, c["block_table"], c["tags"], pairs,
                                                                                               c["seq_lens"])
        self.n, self.q_words = n, c["q"][n:]
        self.q = words_to_tensor(self.q_words, torch, workloads.query_dtype(dtype))
        self.start = torch.tensor([int(x) for x in start], dtype=torch.int32, device="cuda")
        self.clean = [int(x) for x in start]
        mode = lambda t: ekv.MODE_GENERAL if t.any() else ekv.MODE_NATIVE  # noqa: E731
        rows = len(c["seq_lens"])
        part = lambda a, b: ekv.make_batch(self.kv.seq_lens[a:b], self.kv.bt[a:b], self.kv.tags[a:b], None, hq,  # noqa: E731
                                           mode(self.tags[a:b]), int(c["seq_lens"][a:b].max()))
        self.prefixes, self.batch = part(0, n), part(n, rows)

    def decode(self, fp32=True, scale=None, pool=None):
        torch = require_gpu()
        out = torch.full(self.q.shape, float("nan"), dtype=torch.float32 if fp32 else self.q.dtype, device="cuda")
        ws = ekv.decode_shared_workspace(self.kv.pool, self.prefixes, self.batch)
        ws.fill_(0xFF)   # NaN patterns: nothing of it may matter
        ekv.attn_decode_shared(self.kv.pool if pool is None else pool, self.prefixes, self.start, self.batch, self.q, out,
                               default_scale() if scale is None else scale, ws)
        torch.cuda.synchronize()
        return out.double().cpu().numpy()

    def expected(self, s, scale=None):
        p = next((p for p in range(self.n) if self.clean[p] <= s < self.clean[p + 1]), None)
        rows = [(self.table[self.n + s], self.tags[self.n + s], self.own[s])]
        if p is not None:
            rows.insert(0, (self.table[p], self.tags[p], self.prefix[p]))
        return expected_and_bound(self.q_words[s], self.pool, rows, self.dtype, default_scale() if scale is None else scale,
                                  self.hq // self.hkv)

    def check(self, got, sequences, fp32=True, scale=None):
        """fp32: within the arithmetic's bound; 16 bits: and half a step of the type."""
        step = 0.0 if fp32 else (2.0 ** -8 if self.dtype == "bf16" else 2.0 ** -11)
        worst = 0.0
        for s in sequences:
            want, bound = self.expected(s, scale)
            bound = bound + step * (np.abs(want) + bound) + (0.0 if fp32 or self.dtype == "bf16" else 2.0 ** -25)
            off = np.abs(got[s] - want)
            assert (off <= bound).all(), (s, np.nanmax(off - bound), off.max(), bound.max(), np.isnan(off).sum())
            worst = max(worst, float((off / np.maximum(bound, 1e-300)).max()))
        print(f"at most {worst:.3f} of the bound", flush=True)


# ---- to the last bits -----------------------------------------------------------

@pytest.mark.parametrize("fp32", [True, False])
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "e5m2"])
@pytest.mark.parametrize("base", [0.0, 0.5])
@pytest.mark.parametrize("many", [2, 20, 41])
def test_within_the_bound_of_its_arithmetic(many, base, dtype, fp32):
    """Streams (8 columns), one tile (80), tiles and left-over columns (164), values of one sign."""
    print(f"bound: {many} {base} {dtype} {fp32}", flush=True)
    own = np.random.default_rng(many).integers(0, 90, size=many)
    b = Batch([517], own, [0, many], 8, 2, dtype=dtype, base=base, seed=40 + many, positive=True)
    b.check(b.decode(fp32), range(many), fp32)


def test_a_weight_of_8_bits_would_not_pass():
    """The bound tells weights with a remainder from weights without one (the oracle's,
    cut to bf16 as the head of the split is)."""
    b = Batch([517], [40, 3], [0, 2], 8, 2, seed=42, positive=True)
    want, bound = b.expected(0)
    q = encoding.words_to_f64(np.asarray(b.q_words[0], dtype=np.uint16), "bf16")
    k, v = (np.concatenate(x) for x in zip(serve._gather(b.pool, b.table[0], b.tags[0], 517, "bf16"),
                                           serve._gather(b.pool, b.table[1], b.tags[1], 40, "bf16")))
    t = default_scale() * (k[:, 0] @ q[0])
    w = np.exp(t - t.max())
    cut = (w.astype(np.float32).view(np.uint32) & 0xFFFF0000).view(np.float32).astype(np.float64)
    assert (np.abs(cut @ v[:, 0] / w.sum() - want[0]) > bound[0]).any()


# ---- paths ----------------------------------------------------------------------

@pytest.mark.parametrize("dtype,base", [("bf16", 0.0), ("fp16", 0.3), ("e5m2", 0.3)])
@pytest.mark.parametrize("name", list(CASES))
def test_cases_of_their_own_division(name, dtype, base):
    print(f"path: {name} {dtype} {base}", flush=True)
    hq, hkv, prefix, start, own, pick, _ = CASES[name]
    b = Batch(prefix, own, start, hq, hkv, dtype=dtype, base=base, seed=50)
    got = b.decode()
    assert np.isfinite(got).all()
    b.check(got, pick)


@pytest.mark.parametrize("dtype,base", [("bf16", 0.0), ("bf16", 0.5), ("fp16", 0.0), ("e5m2", 0.0), ("e5m2", 0.5)])
@pytest.mark.parametrize("name", list(CASES))
def test_every_token_counts_once(name, dtype, base):
    """At scale 0 every weight is 1, and values of a few whole steps sum exactly in 32 bits:
    what is left is the quotient, 2 roundings, for every sequence.  A token that is lost,
    or counted twice, is off by 1 / n of a value at least."""
    print(f"tokens: {name} {dtype} {base}", flush=True)
    hq, hkv, prefix, start, own, _, _ = CASES[name]
    b = Batch(prefix, own, start, hq, hkv, dtype=dtype, base=base, seed=70, whole=True)
    got = b.decode(scale=0.0)
    total = lambda row, n: serve._gather(b.pool, b.table[row], b.tags[row], int(n), dtype)[1].sum(0) if n else np.zeros((hkv, 128))  # noqa: E731
    sums, tokens = np.stack([total(b.n + s, n) for s, n in enumerate(own)]), np.array(own)
    for p, n in enumerate(prefix):
        sums[start[p]:start[p + 1]] += total(p, n)
        tokens[start[p]:start[p + 1]] += n
    want = (sums / np.maximum(tokens, 1)[:, None, None])[:, :, None].repeat(hq // hkv, 2).reshape(got.shape)
    assert np.abs(sums).max() * 8 < 2**24
    assert (np.abs(got - want) <= 3 * 2.0 ** -24 * np.abs(want)).all()


@pytest.mark.parametrize("dtype", ["bf16", "e5m2"])
@pytest.mark.parametrize("base_of", ["prefix", "own"])
def test_prefixes_and_sequences_in_modes_of_their_own(base_of, dtype):
    """NATIVE prefixes before GENERAL sequences, and the reverse: streams and tiles."""
    print(f"modes: {base_of} {dtype}", flush=True)
    b = Batch([300, 90], [70, 33, 64, 100] * 6, [0, 21, 24], 8, 2, dtype=dtype, base=0.6, base_of=base_of, seed=60)
    assert (b.prefixes.mode, b.batch.mode) == ((ekv.MODE_GENERAL, ekv.MODE_NATIVE) if base_of == "prefix" else
                                               (ekv.MODE_NATIVE, ekv.MODE_GENERAL))
    b.check(b.decode(), range(24))


# ---- arrays that are not as they should be -----------------------------------------

@pytest.mark.parametrize("prefix,start,clean", [
    ([100, 200, 300], [3, 1, 8, 6], [3, 3, 8, 8]), ([100, 200, 300], [2**31 - 1, 0, -2**31, 7], [12] * 4),
    ([100, 200, 300], [-9, -1, 99, 5], [0, 0, 12, 12]), ([70], [7, 2], [7, 7]), ([70], [-3, 4], [0, 4]),
    ([20 + p for p in range(70)], [0, 3, 1] + [2] * 62 + [9, 4, 10, 99, 11, 3], [0, 3, 3] + [3] * 62 + [9, 9, 10, 12, 12, 12])])
def test_boundaries_are_clamped_and_made_nondecreasing(prefix, start, clean):
    """The results are those of the boundaries that the contract makes of them."""
    assert len(start) == len(clean) == len(prefix) + 1
    b = Batch(prefix, [20, 0, 33, 5] * 3, start, 8, 2, seed=61)
    b.clean = clean
    b.check(b.decode(), range(12))


def test_entries_outside_the_pool_read_nothing_behind_it():
    """The pool is the front of a larger array whose other blocks are NaN: entries that
    point there (one past the last, the largest, negative ones), of a prefix and of
    sequences, show no NaN, and sequences that have none are right."""
    torch = require_gpu()
    b = Batch([300, 200], [50] * 20, [0, 10, 20], 16, 2, seed=62)
    blocks = b.kv.kv.shape[0]
    whole = torch.full((2 * blocks, *b.kv.kv.shape[1:]), -1, dtype=torch.int16, device="cuda")   # (0xffff: NaN)
    whole[:blocks] = b.kv.kv
    pool = ekv.make_pool(whole[:blocks], 2)
    for row, col, entry in ((0, 3, blocks), (0, 18, 2**31 - 1), (2 + 12, 0, blocks + 1), (2 + 13, 3, -1), (2 + 14, 2, -2**31)):
        b.kv.bt[row, col] = entry
    got = b.decode(pool=pool)
    assert np.isfinite(got).all()
    b.check(got, [s for s in range(10, 20) if s not in (12, 13, 14)])
