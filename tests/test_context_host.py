"""The long-context entry points without a GPU: their refusals, each before
anything is enqueued, with a message; workspace sizes; the bindings' checks."""

import ctypes

import pytest

from paper_2609_33536_amd import ekv
from tests.test_serve_bindings import Device, calls  # noqa: F401
from tests.test_serve_host import AT, INVALID, ROPE, UNSUPPORTED, _batch, _pool, _refused

torch = pytest.importorskip("torch")
BF, FP, I32 = torch.bfloat16, torch.float16, torch.int32


@pytest.fixture(scope="module")
def lib():
    from __graft_entry__ import _ensure_built
    _ensure_built()
    return ekv.lib()


# ---- norm, rotation and append ---------------------------------------------------

def _norm(**kw):
    a = dict(q_weight=AT, k_weight=AT, q_stride=0, k_stride=128, eps=1e-6, offset=0.0)
    a.update(kw)
    return ekv.HeadNorm(*a.values())


@pytest.mark.parametrize("kw,word", [
    (dict(eps=0.0), "eps"), (dict(eps=-1e-6), "eps"), (dict(eps=1e-31), "eps"), (dict(eps=1e7), "eps"), (dict(eps=float("nan")), "eps"),
    (dict(eps=float("inf")), "eps"), (dict(offset=float("nan")), "offset"), (dict(offset=float("inf")), "offset"),
    (dict(q_stride=64), "stride"), (dict(k_stride=-128), "stride"), (dict(q_stride=132), "stride"), (dict(k_stride=1 << 20), "stride"),
    (dict(q_weight=AT + 8), "aligned"), (dict(k_weight=AT + 2), "aligned")])
def test_norm_refusals(lib, kw, word):
    r = ekv.Rope(AT, 128, 0, 1.0)
    n = _norm(**kw)
    _refused(lib, lib.ekv_norm_rope_append(ctypes.byref(_pool()), ctypes.byref(r), ctypes.byref(n), *ROPE.values(), None), INVALID, word)


@pytest.mark.parametrize("kw,rope,pool,want,word", [
    ({}, dict(turns=None), {}, INVALID, "turns"), ({}, dict(rotary_dim=24), {}, UNSUPPORTED, "rotary_dim"),
    (dict(n=-1), {}, {}, INVALID, "sizes"), (dict(q=None), {}, {}, INVALID, "q"), (dict(k_stride=1016), {}, {}, INVALID, "stride"),
    (dict(v=AT + 8), {}, {}, INVALID, "aligned"), ({}, {}, dict(head_dim=64), UNSUPPORTED, "head_dim")])
def test_norm_rope_append_refuses_what_rope_append_does(lib, kw, rope, pool, want, word):
    r = ekv.Rope(*dict(dict(turns=AT, rotary_dim=128, layout=0, magnitude=1.0), **rope).values())
    n = _norm()
    _refused(lib, lib.ekv_norm_rope_append(ctypes.byref(_pool(**pool)), ctypes.byref(r), ctypes.byref(n), *dict(ROPE, **kw).values(), None),
             want, word)


def test_norm_rope_append_needs_a_norm_and_takes_no_rows(lib):
    r, n = ekv.Rope(AT, 128, 0, 1.0), _norm(q_weight=None, k_weight=None)
    _refused(lib, lib.ekv_norm_rope_append(ctypes.byref(_pool()), ctypes.byref(r), None, *ROPE.values(), None), INVALID, "norm")
    assert lib.ekv_norm_rope_append(ctypes.byref(_pool()), ctypes.byref(r), ctypes.byref(n), *dict(ROPE, n=0, q=None).values(), None) == ekv.OK


@pytest.mark.parametrize("q_weight,k_weight", [((128,), (2, 128)), ((8, 128), (128,)), (None, (128,))])
def test_norm_binding_passes_strides(calls, q_weight, k_weight):  # noqa: F811
    make = lambda s: None if s is None else Device(s, BF)  # noqa: E731
    norm = ekv.make_head_norm(make(q_weight), make(k_weight), 1e-5, 1.0)
    assert norm.q_stride == (128 if q_weight and len(q_weight) == 2 else 0)
    assert norm.k_stride == (128 if len(k_weight) == 2 else 0) and bool(norm.q_weight) == (q_weight is not None)
    rope = ekv.Rope(AT, 128, 0, 1.0)
    x = lambda h: Device((3, h, 128), BF)  # noqa: E731
    ekv.norm_rope_append(_pool(num_kv_heads=2), rope, norm, Device((3,), I32), Device((3,), I32), x(8), x(2), x(2), x(8))
    assert [c[0] for c in calls] == ["ekv_norm_rope_append"]


@pytest.mark.parametrize("weights", [(Device((64,), BF), None), (Device((1, 8, 128), BF), None), (None, Device((128, 2), BF)),
                                     (Device((8, 128), BF, (256, 1)), None)])
def test_norm_weights_that_are_not_rows_of_128(weights):
    with pytest.raises(ekv.EkvError):
        ekv.make_head_norm(*weights)


@pytest.mark.parametrize("q_weight,k_weight", [(Device((128,), FP), None), (Device((4, 128), BF), None), (None, Device((8, 128), BF)),
                                               (None, Device((128,), torch.float32))])
def test_norm_weights_of_another_type_or_number_of_heads(calls, q_weight, k_weight):  # noqa: F811
    x = lambda h: Device((3, h, 128), BF)  # noqa: E731
    with pytest.raises(ekv.EkvError):
        ekv.norm_rope_append(_pool(num_kv_heads=2), ekv.Rope(AT, 128, 0, 1.0), ekv.make_head_norm(q_weight, k_weight),
                             Device((3,), I32), Device((3,), I32), x(8), x(2), x(2), x(8))
    assert not calls


# ---- key bounds, selection, decode ----------------------------------------------

SHAPES = [
    ({}, dict(num_q_heads=24), UNSUPPORTED, "group"), ({}, dict(num_q_heads=20), INVALID, "multiple"),
    ({}, dict(seq_lens=None), INVALID, "seq_lens"), ({}, dict(mode=ekv.MODE_GENERAL), INVALID, "tag"),
    ({}, dict(max_seq_len=129), INVALID, "max_seq_len"), ({}, dict(max_blocks=1 << 26), UNSUPPORTED, "max_blocks"),
    ({}, dict(batch=(1 << 19) + 1), UNSUPPORTED, "2^22"), (dict(head_dim=64), {}, UNSUPPORTED, "head_dim"),
    (dict(dtype=ekv.DTYPE_FP32), {}, UNSUPPORTED, "dtype"), (dict(kv=None), {}, INVALID, "kv")]


@pytest.mark.parametrize("pool,batch,want,word", SHAPES)
def test_refused_shapes(lib, pool, batch, want, word):
    p, b = _pool(**pool), _batch(**batch)
    pp, bp = ctypes.byref(p), ctypes.byref(b)
    _refused(lib, lib.ekv_key_bounds(pp, bp, AT, AT, None), want, word)
    _refused(lib, lib.ekv_select_blocks(pp, bp, AT, AT, 4, 1, 1, AT, AT, AT, 1 << 40, None), want, word)
    _refused(lib, lib.ekv_attn_decode_selected(pp, bp, AT, AT, 4, AT, AT, ekv.DTYPE_FP32, 0.1, AT, 1 << 40, None), want, word)
    assert lib.ekv_select_workspace_bytes(pp, bp, 4) == 0 and lib.ekv_decode_selected_workspace_bytes(pp, bp, 4) == 0


@pytest.mark.parametrize("kw,batch,want,word", [
    (dict(bounds=None), {}, INVALID, "bounds"), (dict(bounds=AT + 8), {}, INVALID, "aligned"),
    ({}, dict(batch=1 << 18, max_blocks=1 << 14), UNSUPPORTED, "too many blocks")])
def test_key_bounds_refusals(lib, kw, batch, want, word):
    a = dict(known=None, bounds=AT)
    a.update(kw)
    _refused(lib, lib.ekv_key_bounds(ctypes.byref(_pool()), ctypes.byref(_batch(**batch)), *a.values(), None), want, word)


SELECT = dict(q=AT, bounds=AT, budget=4, sink=1, recent=1, selected=AT, counts=AT, ws=AT, ws_bytes=1 << 40)


@pytest.mark.parametrize("kw,batch,want,word", [
    (dict(q=None), {}, INVALID, "q"), (dict(bounds=None), {}, INVALID, "bounds"), (dict(selected=None), {}, INVALID, "selected"),
    (dict(counts=None), {}, INVALID, "counts"), (dict(budget=0), {}, INVALID, "budget"), (dict(budget=-1), {}, INVALID, "budget"),
    (dict(budget=1 << 20), {}, UNSUPPORTED, "budget"), (dict(sink=-1), {}, INVALID, "sink"), (dict(recent=-1), {}, INVALID, "recent"),
    (dict(sink=3, recent=2), {}, INVALID, "exceed"), (dict(sink=2 ** 31 - 1, recent=2 ** 31 - 1), {}, INVALID, "exceed"),
    (dict(ws=None), {}, INVALID, "workspace"), (dict(ws_bytes=255), {}, INVALID, "workspace"), (dict(ws=AT + 8), {}, INVALID, "aligned"),
    (dict(q=AT + 4), {}, INVALID, "aligned"), (dict(bounds=AT + 8), {}, INVALID, "aligned"),
    ({}, dict(batch=1 << 16, max_blocks=1 << 14), UNSUPPORTED, "too many blocks")])
def test_select_refusals(lib, kw, batch, want, word):
    _refused(lib, lib.ekv_select_blocks(ctypes.byref(_pool()), ctypes.byref(_batch(**batch)), *dict(SELECT, **kw).values(), None), want, word)


SELECTED = dict(selected=AT, counts=AT, budget=4, q=AT, out=AT, out_dtype=ekv.DTYPE_FP32, scale=0.1, ws=AT, ws_bytes=1 << 40)


@pytest.mark.parametrize("kw,want,word", [
    (dict(selected=None), INVALID, "selected"), (dict(q=None), INVALID, "q"), (dict(out=None), INVALID, "out"),
    (dict(budget=0), INVALID, "budget"), (dict(budget=1 << 20), UNSUPPORTED, "budget"), (dict(out_dtype=ekv.DTYPE_FP16), INVALID, "out_dtype"),
    (dict(scale=float("nan")), INVALID, "scale"), (dict(ws=None), INVALID, "workspace"), (dict(ws_bytes=1024), INVALID, "workspace"),
    (dict(ws=AT + 4), INVALID, "aligned"), (dict(q=AT + 8), INVALID, "aligned"), (dict(out=AT + 2), INVALID, "aligned")])
def test_decode_selected_refusals(lib, kw, want, word):
    _refused(lib, lib.ekv_attn_decode_selected(ctypes.byref(_pool()), ctypes.byref(_batch()), *dict(SELECTED, **kw).values(), None), want, word)


def test_empty_batches_are_nothing(lib):
    b = _batch(batch=0, seq_lens=None, block_table=None)
    pp, bp = ctypes.byref(_pool()), ctypes.byref(b)
    assert lib.ekv_key_bounds(pp, bp, None, None, None) == ekv.OK
    assert lib.ekv_select_blocks(pp, bp, None, None, 4, 1, 1, None, None, None, 0, None) == ekv.OK
    assert lib.ekv_attn_decode_selected(pp, bp, None, None, 4, None, None, ekv.DTYPE_FP32, 0.1, None, 0, None) == ekv.OK
    assert lib.ekv_select_workspace_bytes(pp, bp, 4) > 0 and lib.ekv_decode_selected_workspace_bytes(pp, bp, 4) > 0


@pytest.mark.parametrize("batch,blocks,budget", [(1, 62501, 256), (3, 4097, 1), (64, 2048, 128), (1, 700, 64), (1, 1 << 20, 4096), (2, 64, 64)])
def test_select_workspace_holds_what_any_first_and_newest_blocks_leave(lib, batch, blocks, budget):
    """The size does not ask for sink and recent: it covers all of them."""
    p, b = _pool(), _batch(batch=batch, max_blocks=blocks)
    size = lib.ekv_select_workspace_bytes(ctypes.byref(p), ctypes.byref(b), budget)
    assert 0 < size <= 256 * 3 + batch * 8 * (blocks + 4096) * 12
    for sink, recent in ((0, 0), (1, 0), (0, budget), (budget // 2, budget - budget // 2)):
        a = dict(SELECT, budget=budget, sink=sink, recent=recent, q=AT + 4)   # (refused behind the workspace's check)
        _refused(lib, lib.ekv_select_blocks(ctypes.byref(p), ctypes.byref(b), *dict(a, ws_bytes=size).values(), None), INVALID, "aligned")


@pytest.mark.parametrize("batch,budget,pieces", [(1, 1, 1), (1, 32, 1), (1, 33, 3), (1, 256, 16), (1, 100000, 32), (16, 256, 2),
                                                 (17, 256, 1), (32, 128, 1), (33, 127, 1), (33, 128, 2), (48, 128, 2),
                                                 (49, 128, 1), (500, 16, 1)])
def test_decode_selected_workspace_sizes(lib, batch, budget, pieces):
    p, b = _pool(), _batch(batch=batch)
    size = lib.ekv_decode_selected_workspace_bytes(ctypes.byref(p), ctypes.byref(b), budget)
    slots = 8 * batch * pieces * 4 if pieces > 1 else 0
    align = lambda x: (x + 255) & ~255  # noqa: E731
    assert size == align(align(32768 + slots * 8) + slots * 512)


def _device_batch():
    return _pool(num_kv_heads=2), ekv.Batch(4, 8, 6, ekv.MODE_NATIVE, 0, AT, AT, None, None)


GOOD = dict(bounds=((4, 2, 6, 2, 128), BF), q=((4, 8, 128), BF), selected=((4, 2, 5), I32), counts=((4, 2), I32),
            out=((4, 8, 128), BF), known=((4,), I32))


def _tensors(**kw):
    return {k: None if v is None else Device(*v) for k, v in dict(GOOD, **kw).items()}


def test_bindings_pass_their_tensors_on(calls):  # noqa: F811
    pool, batch = _device_batch()
    ws = Device((1 << 20,), torch.uint8)
    for extra in ({}, dict(bounds=((4, 2, 6, 2, 128), torch.int16)), dict(out=((4, 8, 128), torch.float32))):
        t = _tensors(**extra)
        ekv.key_bounds(pool, batch, t["bounds"], t["known"])
        ekv.select_blocks(pool, batch, t["q"], t["bounds"], t["selected"], t["counts"], ws, 1, 2)
        ekv.attn_decode_selected(pool, batch, t["selected"], t["counts"], t["q"], t["out"], 0.1, ws)
    assert {c[0] for c in calls} == {"ekv_key_bounds", "ekv_select_blocks", "ekv_attn_decode_selected"}
    select = [c[1] for c in calls if c[0] == "ekv_select_blocks"][0]
    assert select[4:7] == (5, 1, 2) and select[10] == 1 << 20
    ekv.key_bounds(pool, batch, _tensors()["bounds"])
    assert calls[-1][1][2] is None
    ekv.attn_decode_selected(pool, batch, _tensors()["selected"], None, _tensors()["q"], _tensors()["out"], 0.1, ws)
    assert calls[-1][1][3] is None and calls[-1][1][4] == 5


@pytest.mark.parametrize("name,bad", [
    ("bounds", ((4, 2, 5, 2, 128), BF)), ("bounds", ((4, 2, 6, 2, 128), FP)), ("bounds", ((4, 2, 6, 2, 128), torch.uint8)),
    ("bounds", ((4, 2, 6, 2, 128), BF, (4000, 1536, 256, 128, 1))), ("bounds", None), ("known", ((3,), I32)), ("known", ((4,), torch.int64)),
    ("q", ((4, 8, 128), FP)), ("q", ((3, 8, 128), BF)), ("q", ((4, 8, 128), BF, (2048, 128, 1))), ("selected", ((4, 3, 5), I32)),
    ("selected", ((4, 2), I32)), ("selected", ((4, 2, 5), torch.int64)), ("selected", None), ("counts", ((4, 3), I32)),
    ("out", ((4, 8, 64), BF)), ("out", ((4, 8, 128), FP)), ("out", None)])
def test_bindings_refuse_what_is_not_the_batch_s(calls, name, bad):  # noqa: F811
    pool, batch = _device_batch()
    t, ws, refused = _tensors(**{name: bad}), Device((1 << 20,), torch.uint8), 0
    for call in (lambda: ekv.key_bounds(pool, batch, t["bounds"], t["known"]),
                 lambda: ekv.select_blocks(pool, batch, t["q"], t["bounds"], t["selected"], t["counts"], ws),
                 lambda: ekv.attn_decode_selected(pool, batch, t["selected"], t["counts"], t["q"], t["out"], 0.1, ws)):
        before = len(calls)
        try:
            call()
        except ekv.EkvError:
            refused += 1
            assert len(calls) == before
    uses = {"bounds": 2, "known": 1, "q": 2, "selected": 2, "counts": 2, "out": 1}[name]
    assert refused == uses


def test_workspace_of_a_refused_shape_says_why(lib):
    with pytest.raises(ekv.EkvError, match="budget"):
        ekv.select_workspace(_pool(), _batch(), 0)
    with pytest.raises(ekv.EkvError, match="group"):
        ekv.decode_selected_workspace(_pool(), _batch(num_q_heads=24), 4)
