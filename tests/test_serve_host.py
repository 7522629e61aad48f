"""The serving-step entry points without a GPU: their refusals, each before
anything is enqueued, with a message; the rotary table against the oracle;
workspace sizes."""

import ctypes

import numpy as np
import pytest

from oracle import serve
from paper_2609_33536_amd import ekv, kvpool

INVALID, UNSUPPORTED = ekv.ERR_INVALID, ekv.ERR_UNSUPPORTED
AT = 0x10000   # a non-NULL, 16-byte aligned address that no refused call reads


@pytest.fixture(scope="module")
def lib():
    from __graft_entry__ import _ensure_built
    _ensure_built()
    return ekv.lib()


def _pool(**kw):
    a = dict(kv=AT, num_blocks=64, num_kv_heads=8, page_size=16, head_dim=128, dtype=ekv.DTYPE_BF16)
    a.update(kw)
    return ekv.Pool(*[a[f] for f, _ in ekv.Pool._fields_])


def _batch(**kw):
    a = dict(batch=4, num_q_heads=32, max_blocks=8, mode=ekv.MODE_NATIVE, max_seq_len=0, seq_lens=AT, block_table=AT,
             tags=None, boundaries=None)
    a.update(kw)
    return ekv.Batch(*[a[f] for f, _ in ekv.Batch._fields_])


def _refused(lib, status, want, word):
    assert status == want, (status, lib.ekv_last_error())
    assert word in lib.ekv_last_error().decode()


EXTEND = dict(batch=2, max_blocks=4, seq_lens=AT, new_lens=AT, start=None, block_table=AT, tags=None, seq_lens_out=AT, cu_q=AT,
              max_tokens=8, slots=AT, positions=AT, status=AT)
LIST = dict(ids=AT, cursor=AT, cursor_out=AT, capacity=16, num_blocks=64)


@pytest.mark.parametrize("kw,ring,want,word", [
    ({}, dict(ids=None), INVALID, "ids"), ({}, dict(cursor=None), INVALID, "cursor"),
    ({}, dict(cursor_out=None), INVALID, "cursor"), ({}, dict(capacity=0), INVALID, "sizes"),
    ({}, dict(num_blocks=0), INVALID, "sizes"), (dict(batch=-1), {}, INVALID, "sizes"),
    (dict(max_blocks=0), {}, INVALID, "sizes"), (dict(max_tokens=-1), {}, INVALID, "sizes"),
    (dict(seq_lens=None), {}, INVALID, "seq_lens"), (dict(block_table=None), {}, INVALID, "block_table"),
    (dict(seq_lens_out=None), {}, INVALID, "seq_lens_out"), (dict(cu_q=None), {}, INVALID, "cu_q"),
    (dict(slots=None), {}, INVALID, "slots"), (dict(status=None), {}, INVALID, "status"),
    (dict(batch=4097), {}, UNSUPPORTED, "4096"), ({}, dict(num_blocks=1 << 27), UNSUPPORTED, "32 bits"),
    (dict(max_blocks=1 << 26), {}, UNSUPPORTED, "32 bits"), (dict(max_tokens=1 << 30), {}, UNSUPPORTED, "32 bits"),
    ({}, dict(capacity=1 << 30), UNSUPPORTED, "32 bits")])
def test_extend_refusals(lib, kw, ring, want, word):
    f = ekv.FreeList(*[dict(LIST, **ring)[n] for n, _ in ekv.FreeList._fields_])
    _refused(lib, lib.ekv_extend(ctypes.byref(f), *dict(EXTEND, **kw).values(), None), want, word)


def test_extend_needs_a_free_list(lib):
    _refused(lib, lib.ekv_extend(None, *EXTEND.values(), None), INVALID, "free list")


ROPE = dict(n=3, positions=AT, slots=AT, q=AT, q_stride=4096, num_q_heads=32, k=AT, k_stride=1024, v=AT, v_stride=1024,
            q_out=AT, q_out_stride=4096)


@pytest.mark.parametrize("kw,rope,pool,want,word", [
    ({}, dict(turns=None), {}, INVALID, "turns"), ({}, dict(rotary_dim=0), {}, UNSUPPORTED, "rotary_dim"),
    ({}, dict(rotary_dim=24), {}, UNSUPPORTED, "rotary_dim"), ({}, dict(rotary_dim=144), {}, UNSUPPORTED, "rotary_dim"),
    ({}, dict(layout=2), {}, INVALID, "layout"), ({}, dict(magnitude=float("nan")), {}, INVALID, "magnitude"),
    (dict(n=-1), {}, {}, INVALID, "sizes"), (dict(num_q_heads=0), {}, {}, INVALID, "sizes"),
    (dict(n=1 << 26), {}, {}, UNSUPPORTED, "tokens"), (dict(num_q_heads=1025), {}, {}, UNSUPPORTED, "heads"),
    (dict(positions=None), {}, {}, INVALID, "positions"), (dict(slots=None), {}, {}, INVALID, "slots"),
    (dict(q=None), {}, {}, INVALID, "q"), (dict(k=None), {}, {}, INVALID, "k"), (dict(v=None), {}, {}, INVALID, "v"),
    (dict(q_out=None), {}, {}, INVALID, "q_out"), (dict(q_stride=4088), {}, {}, INVALID, "stride"),
    (dict(k_stride=1016), {}, {}, INVALID, "stride"), (dict(v_stride=0), {}, {}, INVALID, "stride"),
    (dict(q_out_stride=-4096), {}, {}, INVALID, "stride"), (dict(q_stride=4100), {}, {}, INVALID, "aligned"),
    (dict(q=AT + 2), {}, {}, INVALID, "aligned"), (dict(v=AT + 8), {}, {}, INVALID, "aligned"),
    ({}, {}, dict(kv=None), INVALID, "kv"), ({}, {}, dict(head_dim=64), UNSUPPORTED, "head_dim"),
    ({}, {}, dict(dtype=ekv.DTYPE_FP32), UNSUPPORTED, "dtype")])
def test_rope_append_refusals(lib, kw, rope, pool, want, word):
    r = dict(turns=AT, rotary_dim=128, layout=0, magnitude=1.0)
    r.update(rope)
    r = ekv.Rope(*r.values())
    _refused(lib, lib.ekv_rope_append(ctypes.byref(_pool(**pool)), ctypes.byref(r), *dict(ROPE, **kw).values(), None), want, word)


def test_rope_append_of_no_rows_is_nothing(lib):
    r = ekv.Rope(AT, 128, 0, 1.0)
    assert lib.ekv_rope_append(ctypes.byref(_pool()), ctypes.byref(r), *dict(ROPE, n=0, q=None).values(), None) == ekv.OK


@pytest.mark.parametrize("args,want", [
    (dict(rotary_dim=0), UNSUPPORTED), (dict(rotary_dim=8), UNSUPPORTED), (dict(rotary_dim=256), UNSUPPORTED),
    (dict(base=0.5), INVALID), (dict(base=float("inf")), INVALID), (dict(base=float("nan")), INVALID),
    (dict(scaling="linear", factor=0.5), INVALID), (dict(scaling="base", factor=float("nan")), INVALID),
    (dict(scaling="parts", factor=2.0, context=0.0), INVALID), (dict(scaling="parts", factor=2.0, context=8.0, low=4.0, high=4.0), INVALID),
    (dict(scaling="parts", factor=2.0, context=8.0, low=-1.0), INVALID), (dict(scaling="spiral"), INVALID)])
def test_rope_freqs_refusals(lib, args, want):
    with pytest.raises(ekv.EkvError) as e:
        ekv.rope_freqs(**{"rotary_dim": 128, **args})
    assert e.value.status == want
    assert lib.ekv_rope_freqs(128, 1e4, 9, 1.0, 0.0, 1.0, 4.0, AT) == INVALID
    assert lib.ekv_rope_freqs(128, 1e4, 0, 1.0, 0.0, 1.0, 4.0, None) == INVALID


@pytest.mark.parametrize("rot", [16, 64, 96, 128])
@pytest.mark.parametrize("base", [1.0, 10000.0, 500000.0])
@pytest.mark.parametrize("rule", [{}, dict(scaling="linear", factor=4.0), dict(scaling="base", factor=32.0),
                                  dict(scaling="parts", factor=8.0, context=8192.0, low=1.0, high=4.0)])
def test_rope_freqs_match_the_oracle(lib, rot, base, rule):
    """A table entry is a double rounded down to 2^-64 of a turn: a few roundings of
    2^-53 (the power, the division, the blend) and one unit."""
    got = ekv.rope_freqs(rot, base, **rule)
    want = serve.frequencies(rot, base, **rule) / (2 * serve._PI) * np.longdouble(2) ** 64
    assert got.shape == (rot // 2,)
    assert (np.abs(got.astype(np.longdouble) - want) <= 64 * 2.0 ** -53 * want + 1).all()


SHARED = dict(q=AT, out=AT, out_dtype=ekv.DTYPE_FP32, scale=0.1, ws=AT, ws_bytes=1 << 40)


@pytest.mark.parametrize("kw,prefix,own,start,want,word", [
    (dict(q=None), {}, {}, AT, INVALID, "q and out"), (dict(out=None), {}, {}, AT, INVALID, "q and out"),
    ({}, {}, {}, None, INVALID, "group_start"), (dict(out_dtype=ekv.DTYPE_FP16), {}, {}, AT, INVALID, "out_dtype"),
    (dict(scale=float("inf")), {}, {}, AT, INVALID, "scale"), (dict(ws=None), {}, {}, AT, INVALID, "workspace"),
    (dict(ws_bytes=4096), {}, {}, AT, INVALID, "workspace"), (dict(ws=AT + 4), {}, {}, AT, INVALID, "aligned"),
    (dict(q=AT + 8), {}, {}, AT, INVALID, "aligned"), (dict(out=AT + 2), {}, {}, AT, INVALID, "aligned"),
    ({}, dict(num_q_heads=16), {}, AT, INVALID, "num_q_heads"), ({}, dict(seq_lens=None), {}, AT, INVALID, "seq_lens"),
    ({}, dict(mode=ekv.MODE_GENERAL), {}, AT, INVALID, "tag"), ({}, {}, dict(mode=ekv.MODE_GENERAL), AT, INVALID, "tag"),
    ({}, {}, dict(num_q_heads=24), AT, UNSUPPORTED, "group"), ({}, {}, dict(num_q_heads=20), AT, INVALID, "multiple"),
    ({}, dict(max_seq_len=129), {}, AT, INVALID, "max_seq_len"), ({}, dict(max_blocks=1 << 26), {}, AT, UNSUPPORTED, "max_blocks"),
    ({}, dict(max_blocks=1 << 25), dict(batch=1 << 12), AT, UNSUPPORTED, "too large"),
    ({}, {}, dict(batch=32769, max_blocks=2), AT, UNSUPPORTED, "at most 32768 sequences")])
def test_decode_shared_refusals(lib, kw, prefix, own, start, want, word):
    p, b = _batch(**{"batch": 2, **prefix}), _batch(**own)
    _refused(lib, lib.ekv_attn_decode_shared(ctypes.byref(_pool()), ctypes.byref(p), start, ctypes.byref(b),
                                             *dict(SHARED, **kw).values(), None), want, word)


def test_decode_shared_needs_prefixes_and_takes_an_empty_batch(lib):
    b = _batch()
    _refused(lib, lib.ekv_attn_decode_shared(ctypes.byref(_pool()), None, AT, ctypes.byref(b), *SHARED.values(), None), INVALID,
             "prefixes")
    empty = _batch(batch=0, seq_lens=None, block_table=None)
    assert lib.ekv_attn_decode_shared(ctypes.byref(_pool()), ctypes.byref(b), AT, ctypes.byref(empty),
                                      *dict(SHARED, q=None).values(), None) == ekv.OK
    assert ekv.decode_shared_workspace_bytes(_pool(), _batch(num_q_heads=24), _batch(num_q_heads=24)) == 0


def test_shared_workspace_of_a_larger_batch_serves_a_smaller_one(lib):
    sizes = [ekv.decode_shared_workspace_bytes(_pool(), _batch(batch=p, max_blocks=m), _batch(batch=b, max_blocks=n))
             for p, m, b, n in ((1, 2, 1, 1), (1, 64, 1, 1), (2, 64, 4, 1), (2, 512, 4, 16), (2, 512, 64, 64), (16, 512, 256, 64))]
    assert sizes == sorted(sizes) and sizes[0] > 0
    assert sizes[-1] < 128 << 20


def test_bindings_refuse_wrong_tensors():
    torch = pytest.importorskip("torch")
    i32 = lambda *n: torch.zeros(n, dtype=torch.int32)  # noqa: E731
    for bad in (lambda: ekv.make_free_list(i32(4), i32(3), 8), lambda: ekv.make_free_list(i32(4).long(), i32(2), 8),
                lambda: ekv.make_free_list(i32(4), i32(2), 8),                      # host memory
                lambda: ekv.make_rope(torch.zeros(64, dtype=torch.int64), 128, "spiral"),
                lambda: ekv.make_rope(torch.zeros(32, dtype=torch.int64), 128),
                lambda: ekv.extend(ekv.FreeList(), i32(2), i32(3), i32(2, 4), None, i32(2), i32(3), i32(8), i32(8), i32(4)),
                lambda: ekv.rope_append(_pool(num_kv_heads=2), ekv.Rope(), i32(3), i32(3), torch.zeros((3, 8, 128)),
                                        torch.zeros((3, 2, 128)), torch.zeros((3, 2, 128)), torch.zeros((3, 8, 128))),
                lambda: ekv.attn_decode_shared(_pool(), _batch(batch=2), i32(2), _batch(), None, None, 0.1, None),
                lambda: ekv.attn_decode_shared(_pool(), _batch(batch=2), i32(3).long(), _batch(), None, None, 0.1, None)):
        with pytest.raises(ekv.EkvError) as e:
            bad()
        assert e.value.status == INVALID


def test_binding_refuses_rows_beyond_32_bits():
    class Long:
        def numel(self):
            return (1 << 32) + 1
    torch = pytest.importorskip("torch")
    i32 = lambda *n: torch.zeros(n, dtype=torch.int32)  # noqa: E731
    with pytest.raises(ekv.EkvError) as e:
        ekv.extend(ekv.FreeList(), i32(2), i32(2), i32(2, 4), None, i32(2), i32(3), Long(), None, i32(4))
    assert e.value.status == UNSUPPORTED


@pytest.mark.parametrize("b,new", [(4097, 1), (1100, 1 << 20)])
def test_paged_kv_refuses_what_one_call_cannot_extend_before_its_mirror_changes(b, new):
    kv = object.__new__(kvpool.PagedKV)   # (no device: the refusal comes first)
    kv.mirror = kvpool.HostMirror(np.zeros((b, 1), dtype=np.int32), np.zeros(b, dtype=np.int32), 8, [3, 4, 5])
    with pytest.raises(ekv.EkvError) as e:
        kv.extend(np.full(b, new))
    assert e.value.status == UNSUPPORTED
    assert list(kv.mirror.free) == [3, 4, 5] and not kv.mirror.seq_lens.any()
