"""Decode over shared prefixes on the GPU against the oracle in 64 bits: within
2e-3 absolute (fp32 output) or 2e-3 + 1e-2 |o| (16-bit output), the bound of the
decode tests (probabilities carry 16 significant bits, sums 32)."""

import numpy as np
import pytest

from oracle import fp8 as ofp8
from oracle import serve
from oracle import transitions as otr
from paper_2609_33536_amd import ekv, kvpool, workloads
from tests.gpu_util import check_attention, default_scale, host_safety_check, require_gpu, words_to_tensor

pytestmark = pytest.mark.gpu


def _setup(prefix, own, start, hq, hkv, *, dtype="bf16", base=0.0, placement="random", seed=0, structured=True, spare=3):
    """The state of a shared batch: rows 0 .. P - 1 of one table are the prefixes."""
    torch = require_gpu()
    c = workloads.make_decode_case(list(prefix) + list(own), hq, hkv, seed=seed, base_fraction=base, placement=placement,
                                   dtype=dtype, spare_blocks=spare)
    host_safety_check(c, c["pool"].shape)
    n = len(prefix)
    kv = kvpool.PagedKV(c["pool"], c["block_table"], c["seq_lens"], c["free"], hkv, dtype)
    pool, bt, tags = c["pool"], c["block_table"], c["tags"]
    if len(c["pairs"]):
        kv.demote(c["pairs"], emit_lo=False)
        pool, bt, tags, _, _ = (ofp8 if dtype == "e5m2" else otr).demote(pool, bt, tags, c["pairs"], c["seq_lens"])
    mode = kv.relower()
    bounds = kv.bounds if structured else None
    if mode != ekv.MODE_NATIVE and not structured:
        mode = ekv.MODE_GENERAL

    def part(a, b):
        most = int(c["seq_lens"][a:b].max()) if b > a else 0
        return ekv.make_batch(kv.seq_lens[a:b], kv.bt[a:b], kv.tags[a:b], None if bounds is None else bounds[a:b], hq, mode, most)

    st = dict(kv=kv, prefixes=part(0, n), batch=part(n, len(c["seq_lens"])), q_words=c["q"][n:],
              q=words_to_tensor(c["q"][n:], torch, workloads.query_dtype(dtype)),
              start=torch.tensor(list(start), dtype=torch.int32, device="cuda") if n else None)
    st["oracle"] = lambda scale=None, q=None: serve.decode_shared(
        st["q_words"] if q is None else q, pool, bt[:n], tags[:n], prefix, start, bt[n:], tags[n:], own, dtype, scale)
    return st


def _decode(st, *, fp32=True, scale=None, ws=None, stream=None):
    torch = require_gpu()
    out = torch.full(st["q"].shape, float("nan"), dtype=torch.float32 if fp32 else st["q"].dtype, device="cuda")
    if ws is None:
        ws = ekv.decode_shared_workspace(st["kv"].pool, st["prefixes"], st["batch"])
        ws.fill_(0xFF)   # NaN patterns: nothing of it may matter
    ekv.attn_decode_shared(st["kv"].pool, st["prefixes"], st["start"], st["batch"], st["q"], out,
                           default_scale() if scale is None else scale, ws, stream)
    torch.cuda.synchronize()
    return out


def _run(prefix, own, start, hq, hkv, *, fp32=True, scale=None, **kw):
    print(f"shared: P={len(prefix)} B={len(own)} Hq={hq} Hkv={hkv} fp32={fp32} {kw}", flush=True)
    st = _setup(prefix, own, start, hq, hkv, **kw)
    got = _decode(st, fp32=fp32, scale=scale)
    check_attention(got.float().cpu().numpy(), st["oracle"](scale), fp32)
    return st, got


# ---- one prefix --------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["bf16", "fp16", "e5m2"])
@pytest.mark.parametrize("base", [0.0, 0.5, 1.0])
@pytest.mark.parametrize("group", [1, 2, 4, 8, 16])
def test_groups_types_and_fractions(dtype, base, group):
    """13 sequences: from 13 columns (one wave) to 208 (two tiles) behind a prefix of 17 units."""
    rng = np.random.default_rng(group)
    _run([531], rng.integers(1, 200, size=13), [0, 13], 2 * group, 2, dtype=dtype, base=base, seed=group)


@pytest.mark.parametrize("length", [1, 15, 16, 17, 31, 32, 33, 64, 65, 96, 129, 257, 2048, 2081])
@pytest.mark.parametrize("own", [0, 1, 32, 33])
def test_lengths_around_units(length, own):
    _run([length], [own] * 5 + [1], [0, 6], 16, 2, seed=length)      # 48 columns: tiles
    _run([length], [own, 3], [0, 2], 8, 2, seed=length)              # 8 columns: one wave


@pytest.mark.parametrize("count", [1, 7, 8, 9, 16, 17, 31, 32, 33, 63, 64, 65, 100])
def test_numbers_of_sequences_around_tiles(count):
    """G = 4: 32 columns are 8 sequences, a tile of 128 is 32."""
    rng = np.random.default_rng(count)
    _run([300], rng.integers(0, 70, size=count), [0, count], 8, 2, seed=count, base=0.3)


@pytest.mark.parametrize("dtype", ["bf16", "e5m2"])
@pytest.mark.parametrize("counts", [[40], [41], [33, 40, 8], [72, 9, 34, 1]])
def test_columns_left_over_by_tiles(counts, dtype):
    """G = 4: up to 8 sequences behind full tiles of 32 are streamed (40: one tile and 8
    sequences; 41: two tiles), for one prefix and several."""
    rng = np.random.default_rng(sum(counts))
    start = np.concatenate([[1], 1 + np.cumsum(counts)])
    own = rng.integers(0, 70, size=int(start[-1]) + 2)
    _run(rng.integers(200, 900, size=len(counts)), own, start.tolist(), 8, 2, seed=len(own), base=0.3, dtype=dtype)


@pytest.mark.parametrize("structured", [True, False])
@pytest.mark.parametrize("dtype", ["bf16", "e5m2"])
def test_oldest_half_base_structured_and_general(structured, dtype):
    _run([1024], [200] * 12, [0, 12], 32, 8, dtype=dtype, base=0.5, placement="oldest", structured=structured, fp32=False)


@pytest.mark.parametrize("scale", [-0.3, 0.0, -0.0, 1.0, 0.01])
@pytest.mark.parametrize("dtype", ["bf16", "e5m2"])
def test_softmax_scales(scale, dtype):
    _run([200, 70], [33, 0, 90, 64, 17], [0, 4, 5], 16, 2, scale=scale, dtype=dtype, base=0.5, seed=31)


# ---- several prefixes --------------------------------------------------------

@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("base", [0.0, 0.4])
def test_ragged_groups_of_all_kinds(dtype, base):
    """Groups of 0, 1, 3, 12 and 40 sequences behind prefixes from none to 1500 tokens,
    and sequences in front of and behind all groups."""
    counts, prefix = [3, 0, 1, 12, 0, 40, 1], [700, 64, 33, 1500, 0, 257, 0]
    start = np.concatenate([[2], 2 + np.cumsum(counts)])
    own = np.random.default_rng(5).integers(0, 150, size=int(start[-1]) + 3)
    own[[0, 4, 8]] = 0
    _run(prefix, own, start.tolist(), 16, 4, dtype=dtype, base=base, seed=6)


@pytest.mark.parametrize("groups,per", [(65, 1), (130, 2), (70, 9)])
def test_many_prefixes(groups, per):
    """More than 64 prefixes (a wave scans 64 at a time), few-column and tile kinds."""
    rng = np.random.default_rng(groups)
    _run(rng.integers(0, 90, size=groups), rng.integers(0, 40, size=groups * per), (per * np.arange(groups + 1)).tolist(), 8, 2, seed=7)


def test_many_sequences():
    """More than 512 sequences (lengths are summed 512 at a time)."""
    rng = np.random.default_rng(70)
    _run([100, 40], rng.integers(0, 50, size=700), [10, 600, 690], 2, 2, seed=8)


def test_no_prefix_at_all():
    torch = require_gpu()
    st = _setup([], [100, 0, 33, 1], [], 8, 2, base=0.5, seed=9)
    st["prefixes"] = ekv.make_batch(torch.empty(0, dtype=torch.int32, device="cuda"), torch.empty((0, 2), dtype=torch.int32, device="cuda"),
                                    torch.empty((0, 2), dtype=torch.uint8, device="cuda"), None, 8, ekv.MODE_GENERAL)
    check_attention(_decode(st).cpu().numpy(), st["oracle"](), True)


def test_nothing_anywhere_yields_zeros():
    st = _setup([0, 0], [0, 0, 0], [0, 2, 3], 8, 2, spare=3)
    assert not _decode(st).any()


def test_equals_decode_without_a_prefix():
    """Behind an empty prefix the call computes what ekv_attn_decode does (both within
    half their bound of the same value)."""
    torch = require_gpu()
    st = _setup([0], [300, 17, 512], [0, 3], 8, 2, base=0.5, seed=10)
    got = _decode(st)
    out = torch.empty_like(got)
    ekv.attn_decode(st["kv"].pool, st["batch"], st["q"], out, default_scale(), ekv.decode_workspace(st["kv"].pool, st["batch"]))
    torch.cuda.synchronize()
    assert (got - out).abs().max().item() <= 2e-3


# ---- hard values -------------------------------------------------------------

@pytest.mark.parametrize("where", ["prefix", "own"])
@pytest.mark.parametrize("many", [2, 20])
def test_one_part_outweighs_the_other(where, many):
    """Keys of one part parallel to the queries: its weights are 2^40 times the other's,
    and late in the part (the running maximum rises after output has been summed)."""
    prefix, own = [900], [200] * many
    st = _setup(prefix, own, [0, many], 8, 2, seed=11)
    torch = require_gpu()
    kv, bt = st["kv"].kv, st["kv"].bt
    big = (8.0 * st["q"][:, 0].float()).bfloat16().view(torch.int16)   # query head 0 of each sequence
    words = st["kv"].kv.view(torch.int16)
    rows = [(0, 880, 0)] if where == "prefix" else [(1 + s, 150, s) for s in range(many)]
    for row, tok, s in rows:
        words[bt[row, tok // 16].long(), 0, 0, tok % 16] = big[s]
    torch.cuda.synchronize()
    host = kv.cpu().numpy().view(np.uint16)
    tb, tg = st["kv"].bt.cpu().numpy(), st["kv"].tags.cpu().numpy()
    want = serve.decode_shared(st["q_words"], host, tb[:1], tg[:1], prefix, [0, many], tb[1:], tg[1:], own, "bf16")
    check_attention(_decode(st).cpu().numpy(), want, True)


def test_infinite_scores_in_one_unit_weigh_nothing():
    """A unit all of whose scores are -inf (keys of -inf against positive queries) takes no
    weight: the other units' result stands."""
    torch = require_gpu()
    for many in (2, 20):
        st = _setup([96], [40] * many, [0, many], 8, 2, seed=12)
        q = st["q"].abs().clamp(min=0.01)
        st["q"] = q
        words = q.view(torch.int16).cpu().numpy().view(np.uint16)
        kv = st["kv"].kv.view(torch.int16)
        bt = st["kv"].bt
        for i in range(2):   # the prefix's first unit
            kv[bt[0, i].long(), 0] = torch.tensor(-128, dtype=torch.int16)   # 0xff80: -inf in bf16
        torch.cuda.synchronize()
        host = st["kv"].kv.cpu().numpy().view(np.uint16)
        tb, tg = st["kv"].bt.cpu().numpy(), st["kv"].tags.cpu().numpy()
        want = serve.decode_shared(words, host, tb[:1], tg[:1], [96], [0, many], tb[1:], tg[1:], [40] * many, "bf16")
        assert np.isfinite(want).all()
        check_attention(_decode(st).cpu().numpy(), want, True)


# ---- the call ----------------------------------------------------------------

def test_boundaries_outside_the_batch_are_clamped():
    """Boundaries that fall, or lie outside the batch, are clamped and made nondecreasing."""
    torch = require_gpu()
    prefix, own = [100, 200, 300], [20] * 12
    st = _setup(prefix, own, [0, 4, 4, 12], 8, 2, seed=13)
    want = st["oracle"]()
    st["start"] = torch.tensor([-5, 4, 2, 99], dtype=torch.int32, device="cuda")
    check_attention(_decode(st).cpu().numpy(), want, True)
    st["start"] = torch.tensor([2**31 - 1, 0, -2**31, 7], dtype=torch.int32, device="cuda")   # no group has any sequence
    assert torch.isfinite(_decode(st)).all()


def test_workspace_edges():
    """The exact size between canary bytes; a smaller batch in a larger one's workspace."""
    torch = require_gpu()
    st = _setup([600, 50], [100] * 20, [0, 18, 20], 16, 2, seed=14)
    size = ekv.decode_shared_workspace_bytes(st["kv"].pool, st["prefixes"], st["batch"])
    whole = torch.full((size + 8192,), 0x5A, dtype=torch.uint8, device="cuda")
    got = _decode(st, ws=whole[4096:4096 + size])
    check_attention(got.cpu().numpy(), st["oracle"](), True)
    assert (whole[:4096] == 0x5A).all() and (whole[4096 + size:] == 0x5A).all()
    with pytest.raises(ekv.EkvError):
        _decode(st, ws=whole[4096:4096 + size - 1])
    small = _setup([40], [10, 3], [0, 2], 8, 2, seed=15)
    check_attention(_decode(small, ws=whole).cpu().numpy(), small["oracle"](), True)


@pytest.mark.parametrize("dtype", ["bf16", "e5m2"])
def test_calls_repeat_bit_for_bit_on_other_streams_and_from_a_graph(dtype):
    torch = require_gpu()
    counts = [9, 2, 30]
    start = [0, 9, 11, 41]
    st = _setup([1000, 333, 90], np.random.default_rng(3).integers(0, 300, size=sum(counts)), start, 16, 4, dtype=dtype, base=0.5,
                seed=16)
    ref = _decode(st)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(8):
        assert torch.equal(_decode(st), ref)
        assert torch.equal(_decode(st, stream=side), ref)
    ws = ekv.decode_shared_workspace(st["kv"].pool, st["prefixes"], st["batch"])
    out = torch.empty_like(ref)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ekv.attn_decode_shared(st["kv"].pool, st["prefixes"], st["start"], st["batch"], st["q"], out, default_scale(), ws)
    for replay in range(4):
        st["q"].copy_(torch.randn(st["q"].shape, device="cuda"))
        st["start"].copy_(torch.tensor([0, 9 + replay, 11, 41], dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        assert torch.equal(_decode(st), got)


def test_two_calls_at_once_with_their_own_workspaces():
    torch = require_gpu()
    a = _setup([800], [100] * 30, [0, 30], 16, 2, seed=17)
    b = _setup([500, 60], [40] * 9, [0, 3, 9], 32, 8, seed=18, base=0.5)
    want = [_decode(a), _decode(b)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    spaces = [ekv.decode_shared_workspace(x["kv"].pool, x["prefixes"], x["batch"]) for x in (a, b)]
    for _ in range(6):
        outs = [torch.empty_like(w) for w in want]
        torch.cuda.synchronize()
        for st, s, ws, out in zip((a, b), streams, spaces, outs):
            ekv.attn_decode_shared(st["kv"].pool, st["prefixes"], st["start"], st["batch"], st["q"], out, default_scale(), ws, s)
        torch.cuda.synchronize()
        assert all(torch.equal(o, w) for o, w in zip(outs, want))


def test_table_entries_outside_the_pool_stay_inside_it():
    """Entries past the pool are clamped into it: canary blocks behind it (NaN) do not
    show, and the sequences whose entries are valid are right."""
    torch = require_gpu()
    st = _setup([300], [50] * 10, [0, 10], 16, 2, seed=19)
    want = st["oracle"]()
    st["kv"].bt[3, 1] = st["kv"].mirror.num_blocks + 5
    st["kv"].bt[4, 0] = -3
    got = _decode(st).cpu().numpy()
    ok = [s for s in range(10) if s not in (2, 3)]
    check_attention(got[ok], want[ok], True)


def test_debug_mode_names_a_violation(monkeypatch):
    torch = require_gpu()
    st = _setup([300], [50] * 3, [0, 3], 16, 2, seed=20)
    monkeypatch.setenv("EKV_DEBUG", "1")
    ref = _decode(st)
    st["kv"].bt[0, 2] = -3
    torch.cuda.synchronize()
    with pytest.raises(ekv.EkvError, match="outside the pool"):
        _decode(st)
    assert torch.isfinite(ref).all()


def test_8b_layer_behind_one_long_prefix():
    """64 sequences, 32 / 8 heads, 4096 shared tokens: the oracle's sequences 0, 31 and 63."""
    rng = np.random.default_rng(21)
    prefix, own = [4100], rng.integers(1, 200, size=64)
    torch = require_gpu()
    c = workloads.make_decode_case(prefix + own.tolist(), 32, 8, seed=21, base_fraction=0.5)
    kv = kvpool.PagedKV(c["pool"], c["block_table"], c["seq_lens"], c["free"], 8)
    kv.demote(c["pairs"], emit_lo=False)
    mode = kv.relower()
    pool, bt, tags, _, _ = otr.demote(c["pool"], c["block_table"], c["tags"], c["pairs"], c["seq_lens"])
    part = lambda a, b: ekv.make_batch(kv.seq_lens[a:b], kv.bt[a:b], kv.tags[a:b], kv.bounds[a:b], 32, mode)  # noqa: E731
    q = words_to_tensor(c["q"][1:], torch, "bf16")
    out = torch.empty_like(q)
    pre, bat = part(0, 1), part(1, 65)
    ekv.attn_decode_shared(kv.pool, pre, torch.tensor([0, 64], dtype=torch.int32, device="cuda"), bat, q, out, default_scale(),
                           ekv.decode_shared_workspace(kv.pool, pre, bat))
    torch.cuda.synchronize()
    pick = [0, 31, 63]
    want = serve.decode_shared(c["q"][1:][pick], pool, bt[:1], tags[:1], prefix, [0, 3], bt[1:][pick], tags[1:][pick],
                               own[pick], "bf16")
    check_attention(out.float().cpu().numpy()[pick], want, False)
