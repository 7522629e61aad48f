"""Workspaces of block selection and of the selected decode without a GPU: one that is made
for the largest batch, length and budget serves every smaller call."""

import ctypes
import itertools

import pytest

from paper_2609_33536_amd import ekv
from tests.test_context_host import SELECT, SELECTED, lib  # noqa: F401
from tests.test_serve_host import AT, INVALID, _batch, _pool, _refused

BATCHES = [*range(1, 70), 96, 128, 200, 333, 512]
BLOCKS = [1, 2, 31, 64, 65, 255, 256, 257, 511, 513, 700, 1023, 1025, 1500, 2048, 2049, 4095, 4096, 4097, 4600, 8192, 12289, 62501]
BUDGETS = [1, 2, 63, 128, 256, 257, 1000, 4096, 5000]


def _select_bytes(lib, pool, batch, blocks, budget, stated=0):  # noqa: F811
    b = _batch(batch=batch, max_blocks=blocks, max_seq_len=stated)
    return lib.ekv_select_workspace_bytes(ctypes.byref(pool), ctypes.byref(b), budget)


@pytest.mark.parametrize("hkv", [1, 3, 8])
def test_selection_sizes_never_fall(lib, hkv):  # noqa: F811
    pool = _pool(num_kv_heads=hkv)
    table = {}
    for b, n, k in itertools.product(BATCHES, BLOCKS, BUDGETS):
        bt = _batch(batch=b, max_blocks=n, num_q_heads=4 * hkv, max_seq_len=0)
        table[b, n, k] = lib.ekv_select_workspace_bytes(ctypes.byref(pool), ctypes.byref(bt), k)
        assert table[b, n, k] > 0
    for names, axis in ((BATCHES, 0), (BLOCKS, 1), (BUDGETS, 2)):
        for small, large in zip(names, names[1:]):
            for key, size in table.items():
                if key[axis] == small:
                    other = key[:axis] + (large,) + key[axis + 1:]
                    assert size <= table[other], (key, other)


def test_selection_sizes_are_small_beside_the_bounds(lib):  # noqa: F811
    """12 bytes a block, where its bounds have 256 or 512: chunks of c blocks, fewer than the row's n and at most 4096, keep
    at most ceil(n / c) c < n + c of them."""
    pool = _pool()
    for b, n, k in itertools.product(BATCHES, BLOCKS, BUDGETS):
        assert _select_bytes(lib, pool, b, n, k) <= 1024 + b * 8 * (n + min(n, 4096)) * 12


def test_selection_sizes_by_the_stated_length(lib):  # noqa: F811
    pool = _pool()
    sizes = [_select_bytes(lib, pool, 8, 8192, 128, 16 * n) for n in range(64, 8193, 64)]
    assert sizes == sorted(sizes) and sizes[-1] == _select_bytes(lib, pool, 8, 8192, 128)


@pytest.mark.parametrize("batch,blocks,budget", [(64, 2048, 128), (32, 8192, 256), (8, 62501, 256), (1, 5000, 4096)])
def test_a_selection_workspace_serves_every_smaller_call(lib, batch, blocks, budget):  # noqa: F811
    pool = _pool()
    size = _select_bytes(lib, pool, batch, blocks, budget)
    for b, n, k, sink in itertools.product([x for x in BATCHES if x <= batch], [x for x in BLOCKS if x <= blocks], [x for x in BUDGETS if x <= budget],
                                           (0, 1)):
        bt = _batch(batch=b, max_blocks=blocks, max_seq_len=16 * n)
        a = dict(SELECT, budget=k, sink=sink, recent=0, q=AT + 4, ws_bytes=size)   # (refused behind the workspace's check)
        _refused(lib, lib.ekv_select_blocks(ctypes.byref(pool), ctypes.byref(bt), *a.values(), None), INVALID, "aligned")


@pytest.mark.parametrize("hkv,group", [(8, 4), (1, 16), (8, 16)])
def test_every_reported_decode_workspace_is_taken_for_every_batch(lib, hkv, group):  # noqa: F811
    pool = _pool(num_kv_heads=hkv)
    sizes = {}
    for b, k in itertools.product(BATCHES, (1, 33, 128, 256, 1000)):
        bt = _batch(batch=b, max_blocks=1024, num_q_heads=group * hkv)
        sizes[b, k] = lib.ekv_decode_selected_workspace_bytes(ctypes.byref(pool), ctypes.byref(bt), k)
    for size in set(sizes.values()):
        for b, k in itertools.product(BATCHES, (1, 128, 1000)):
            bt = _batch(batch=b, max_blocks=1024, num_q_heads=group * hkv)
            a = dict(SELECTED, budget=k, q=AT + 4, ws_bytes=size)   # (refused behind the workspace's check)
            _refused(lib, lib.ekv_attn_decode_selected(ctypes.byref(pool), ctypes.byref(bt), *a.values(), None), INVALID, "aligned")
    bt = _batch(batch=1, max_blocks=1024, num_q_heads=group * hkv)
    _refused(lib, lib.ekv_attn_decode_selected(ctypes.byref(pool), ctypes.byref(bt), *dict(SELECTED, ws_bytes=min(sizes.values()) - 1).values(), None),
             INVALID, "workspace")


@pytest.mark.parametrize("hkv", [1, 3, 8, 64])
def test_the_binding_s_workspace_has_room_for_smaller_batches_in_full(lib, hkv):  # noqa: F811
    pool = _pool(num_kv_heads=hkv)
    for budget in (16, 150, 700):
        most = 0
        for b in [*range(1, 70), 96, 128, 129, 256, 257, 384, 385, 600]:
            batch = _batch(batch=b, num_q_heads=4 * hkv, max_blocks=1024)
            most = max(most, ekv.decode_selected_workspace_bytes(pool, batch, budget))
            assert ekv.decode_selected_workspace(pool, batch, budget, device="cpu").numel() >= most
            assert batch.batch == b
