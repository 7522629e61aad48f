"""What the serving-step bindings refuse and take, without a GPU: the tensors are
stand-ins that claim to lie on the device, and the library is a stand-in too."""

import ctypes

import pytest

from paper_2609_33536_amd import ekv

torch = pytest.importorskip("torch")
AT = 0x10000


class Device:
    """A tensor's shape, type and strides, on the device, with no memory behind them."""
    is_cuda = True

    def __init__(self, shape, dtype, stride=None):
        t = torch.empty(shape, dtype=dtype, device="meta") if stride is None else torch.empty_strided(shape, stride, dtype=dtype, device="meta")
        self.t, self.shape, self.dtype = t, t.shape, dtype

    def __getattr__(self, name):
        return getattr(self.t, name)

    def data_ptr(self):
        return AT


@pytest.fixture
def calls(monkeypatch):
    seen = []

    class Lib:
        def __getattr__(self, name):
            return lambda *a: seen.append((name, a)) or ekv.OK
    monkeypatch.setattr(ekv, "lib", Lib)
    monkeypatch.setattr(ekv, "_stream", lambda s: 0)
    return seen


def _pool(dtype=ekv.DTYPE_BF16, hkv=2):
    return ekv.Pool(AT, 64, hkv, 16, 128, dtype)


def _batch(b, hq=8):
    return ekv.Batch(b, hq, 8, ekv.MODE_NATIVE, 0, AT, AT, None, None)


BF, FP, F4 = torch.bfloat16, torch.float16, torch.float32


@pytest.mark.parametrize("pool,q,out", [
    (ekv.DTYPE_BF16, ((3, 8, 128), BF), ((4, 8, 128), BF)), (ekv.DTYPE_BF16, ((4, 4, 128), BF), ((4, 8, 128), BF)),
    (ekv.DTYPE_BF16, ((4, 8, 128), BF), ((3, 8, 128), BF)), (ekv.DTYPE_BF16, ((4, 8, 128), BF), ((4, 8, 64), F4)),
    (ekv.DTYPE_BF16, ((4, 8, 128), F4), ((4, 8, 128), F4)), (ekv.DTYPE_BF16, ((4, 8, 128), FP), ((4, 8, 128), BF)),
    (ekv.DTYPE_FP16, ((4, 8, 128), BF), ((4, 8, 128), FP)), (ekv.DTYPE_E5M2, ((4, 8, 128), BF), ((4, 8, 128), FP)),
    (ekv.DTYPE_FP16, ((4, 8, 128), FP), ((4, 8, 128), BF)), (ekv.DTYPE_E5M2, ((4, 8, 128), FP), ((4, 8, 128), torch.float64)),
    (ekv.DTYPE_BF16, ((8, 4, 128), BF), ((4, 8, 128), BF)), (ekv.DTYPE_BF16, ((0, 8, 128), BF), ((4, 8, 128), BF))])
def test_decode_shared_refuses_queries_and_outputs_that_are_not_the_batch_s(calls, pool, q, out):
    with pytest.raises(ekv.EkvError) as e:
        ekv.attn_decode_shared(_pool(pool), _batch(2), Device((3,), torch.int32), _batch(4), Device(*q), Device(*out), 0.1,
                               Device((64,), torch.uint8))
    assert e.value.status == ekv.ERR_INVALID and not calls


@pytest.mark.parametrize("pool,q", [(ekv.DTYPE_BF16, BF), (ekv.DTYPE_FP16, FP), (ekv.DTYPE_E5M2, FP)])
@pytest.mark.parametrize("fp32", [False, True])
def test_decode_shared_takes_the_batch_s(calls, pool, q, fp32):
    ekv.attn_decode_shared(_pool(pool), _batch(2), Device((3,), torch.int32), _batch(4), Device((4, 8, 128), q),
                           Device((4, 8, 128), F4 if fp32 else q), 0.1, Device((64,), torch.uint8))
    assert [name for name, _ in calls] == ["ekv_attn_decode_shared"]


def _turn(hq, hkv, n, q=None, k=None, v=None, out=None):
    dense = lambda h, s=None: Device((n, h, 128), BF, s)  # noqa: E731
    ekv.rope_append(_pool(hkv=hkv), ekv.Rope(AT, 128, 0, 1.0), Device((n,), torch.int32), Device((n,), torch.int32),
                    dense(hq, q), dense(hkv, k), dense(hkv, v), dense(hq, out))


@pytest.mark.parametrize("n", [1, 5])
def test_rope_append_takes_a_single_head_whatever_its_stride(calls, n):
    """The stride between heads says nothing where there is one: [1][n][128] transposed, say."""
    _turn(4, 1, n, k=(256, 128 * n, 1), v=(128, 999, 1))
    _turn(1, 1, n, q=(384, 384, 1), k=(384, 0, 1), v=(384, 384, 1), out=(128, 7, 1))
    strides = [[a[6], a[9], a[11], a[13]] for _, a in calls]
    if n > 1:   # (of a single row the stride says nothing either)
        assert strides == [[512, 256, 128, 512], [384, 384, 384, 128]]
    else:
        assert strides == [[512, 128, 128, 512], [128] * 4]


@pytest.mark.parametrize("bad", [dict(q=(512, 64, 1)), dict(k=(512, 256, 1)), dict(v=(512, 128, 2)), dict(out=(512, 0, 1))])
def test_rope_append_refuses_heads_that_are_not_packed(calls, bad):
    with pytest.raises(ekv.EkvError) as e:
        _turn(4, 2, 5, **bad)
    assert e.value.status == ekv.ERR_INVALID and not calls
