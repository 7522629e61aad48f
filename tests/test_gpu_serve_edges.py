"""Calls of the serving step at the edges of what is allowed: views whose strides say
nothing, a device that parts from its mirror, other streams, graphs that share scratch."""

import numpy as np
import pytest

from paper_2609_33536_amd import ekv, kvpool, workloads
from tests.gpu_util import default_scale, require_gpu
from tests.test_gpu_decode_shared_paths import Batch

pytestmark = pytest.mark.gpu


def test_rope_append_of_single_heads_and_single_rows_in_any_view():
    torch = require_gpu()
    turns = torch.from_numpy(ekv.rope_freqs(128).view(np.int64)).cuda()
    rope = ekv.make_rope(turns, 128)
    for n in (1, 9):
        gen = torch.Generator(device="cuda")
        gen.manual_seed(n)
        make = lambda *shape: torch.randn(shape, generator=gen, device="cuda").bfloat16()  # noqa: E731
        q, k, v = make(n, 4, 128), make(n, 1, 128), make(n, 1, 128)
        pos = torch.arange(n, dtype=torch.int32, device="cuda") + 70
        slots = torch.arange(n, dtype=torch.int32, device="cuda")

        def call(q, k, v):
            kv = torch.zeros((2, 2, 1, 16, 128), dtype=torch.int16, device="cuda")
            out = torch.full((n, 4, 128), float("nan"), dtype=torch.bfloat16, device="cuda")
            ekv.rope_append(ekv.make_pool(kv, 1), rope, pos, slots, q, k, v, out)
            torch.cuda.synchronize()
            return kv, out
        want = call(q, k, v)
        assert want[0].any()
        views = [(q, k.reshape(1, n, 128).transpose(0, 1), v.reshape(1, n, 128).transpose(0, 1)),
                 (q, k.as_strided((n, 1, 128), (128, 8, 1)), v.as_strided((n, 1, 128), (128, 0, 1)))]
        if n == 1:
            views.append((q.as_strided((1, 4, 128), (515, 128, 1)), k.as_strided((1, 1, 128), (3, 1, 1)), v))
        for view in views:
            got = call(*view)
            assert all(torch.equal(a, b) for a, b in zip(got, want))


def _kv(seed=0, lens=(20, 64, 0, 33)):
    c = workloads.make_decode_case(list(lens), 8, 2, seed=seed, spare_blocks=40)
    table = np.concatenate([c["block_table"], np.zeros((len(lens), 12), dtype=np.int32)], axis=1)
    return kvpool.PagedKV(c["pool"], table, c["seq_lens"], c["free"], 2)


def test_an_extension_that_the_device_refuses_is_told(monkeypatch):
    """Lengths on the device that were changed behind the mirror: nothing is taken, the
    status says why, and with EKV_DEBUG=1 the call raises and the mirror stays."""
    torch = require_gpu()
    kv = _kv()
    kv.seq_lens[1] = 10**6
    lens, free = kv.mirror.seq_lens.copy(), list(kv.mirror.free)
    monkeypatch.setenv("EKV_DEBUG", "1")
    with pytest.raises(ekv.EkvError, match="took nothing"):
        kv.extend([3, 1, 20, 0])
    assert (kv.mirror.seq_lens == lens).all() and list(kv.mirror.free) == free
    monkeypatch.delenv("EKV_DEBUG")
    _, slots, _ = kv.extend([3, 1, 20, 0])
    assert kv.extend_status.tolist()[0] == ekv.EXTEND_ROW and (slots == -1).all()
    kv = _kv()
    monkeypatch.setenv("EKV_DEBUG", "1")
    _, slots, _ = kv.extend([3, 1, 20, 0])
    assert kv.extend_status.tolist()[:3] == [0, 24, 3] and (slots >= 0).all()
    torch.cuda.synchronize()
    assert (kv.seq_lens.cpu().numpy() == kv.mirror.seq_lens).all() and (kv.bt.cpu().numpy() == kv.mirror.bt).all()


@pytest.mark.parametrize("new", [(3, 1, 20, 0), (0, 0, 0, 0), (45, 60, 128, 100)])
def test_extensions_on_another_stream(new):
    torch = require_gpu()
    want, kv, side = _kv(), _kv(), torch.cuda.Stream()
    a = want.extend(new)
    torch.cuda.synchronize()
    b = kv.extend(new, stream=side)
    side.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    for x, y in ((want.bt, kv.bt), (want.seq_lens, kv.seq_lens), (want.tags, kv.tags)):
        assert torch.equal(x, y)
    assert (kv.mirror.bt == kv.bt.cpu().numpy()).all() and (kv.mirror.seq_lens == kv.seq_lens.cpu().numpy()).all()


def test_graphs_that_share_a_workspace():
    """Two captured calls of different batches over one workspace, replayed in turn on one
    stream with eager calls between: what one leaves there does not reach the other."""
    torch = require_gpu()
    batches = [Batch([700, 33], [40, 0, 90] * 7, [0, 12, 21], 16, 4, base=0.4, seed=80),
               Batch([90], [200, 3], [0, 2], 8, 2, seed=81)]
    want = [b.decode() for b in batches]
    space = lambda b: ekv.decode_shared_workspace(b.kv.pool, b.prefixes, b.batch)  # noqa: E731
    ws = max((space(b) for b in batches), key=lambda t: t.numel())
    outs = [torch.empty(b.q.shape, dtype=torch.float32, device="cuda") for b in batches]
    graphs = []
    for b, out in zip(batches, outs):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            ekv.attn_decode_shared(b.kv.pool, b.prefixes, b.start, b.batch, b.q, out, default_scale(), ws)
        graphs.append(g)
    for replay in range(4):
        for i in (0, 1, 1, 0):
            outs[i].fill_(float("nan"))
            graphs[i].replay()
            if replay % 2:
                torch.cuda.synchronize()
            assert np.array_equal(outs[i].double().cpu().numpy(), want[i])
        assert np.array_equal(batches[replay % 2].decode(), want[replay % 2])
