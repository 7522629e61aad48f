"""Rotary append on the GPU against the oracle in 64 bits.

Tolerance.  The phase is exact to 2^-33 of a turn and the table to a few 2^-53 of
an angle of less than 2^31 radians (below 1e-6 even there); cosine and sine follow
in 32 bits (argument, polynomial and magnitude: under 2^-22), and a turned element
is two products and a sum in 32 bits: in all at most 2^-20 magnitude (|x| + |y|).
Its one rounding to the output adds half a step, eps / 2 of the value, or half the
smallest subnormal."""

import numpy as np
import pytest

from oracle import encoding, fp8, serve
from oracle import transitions as otr
from paper_2609_33536_amd import ekv, workloads
from tests.gpu_util import require_gpu

pytestmark = pytest.mark.gpu
HALF_STEP = {"bf16": (2.0 ** -8, 2.0 ** -134), "fp16": (2.0 ** -11, 2.0 ** -25), "e5m2": (2.0 ** -3, 2.0 ** -17)}


def _torch_dtype(torch, dtype):
    return torch.bfloat16 if dtype == "bf16" else torch.float16


def _values(words, dtype):
    return fp8.bytes_to_f64(words) if dtype == "e5m2" else encoding.words_to_f64(words, dtype)


def _check(got, want, size, dtype):
    """size: magnitude (|x| + |y|) of each element's pair, 0 where it passes through"""
    rel, sub = HALF_STEP[dtype]
    off = np.abs(got - want)
    bound = 2.0 ** -20 * size + rel * (np.abs(want) + 2.0 ** -20 * size) + sub
    bad = ~(off <= bound)
    assert not bad.any(), (f"{bad.sum()} off; worst {np.max(off / np.maximum(bound, 1e-300)):.3f} of the bound; "
                           f"first at {np.argwhere(bad)[0]}: {got[bad][0]} for {want[bad][0]}")


def _pair_size(x, rot, layout, magnitude):
    a = np.abs(x)
    first = np.arange(rot // 2) if layout == "half" else 2 * np.arange(rot // 2)
    second = first + (rot // 2 if layout == "half" else 1)
    out = np.zeros_like(a)
    out[..., first] = out[..., second] = abs(magnitude) * (a[..., first] + a[..., second])
    return out


def _run(n, hq, hkv, *, dtype="bf16", rot=128, layout="half", magnitude=1.0, positions=None, rule=None, packed=False,
         in_place=False, seed=0, skip=(), spread=1.0, nb=None, stream=None):
    torch = require_gpu()
    rng = np.random.default_rng(seed)
    act = workloads.query_dtype(dtype)
    rule = dict(base=10000.0) if rule is None else rule
    theta = serve.frequencies(rot, **rule)
    positions = rng.integers(0, 1 << 20, size=n) if positions is None else np.asarray(positions)
    nb = n // 16 + 4 if nb is None else nb
    slots = rng.permutation(nb * 16)[:n].astype(np.int32)
    for i, value in skip:
        slots[i] = value
    x = {k: workloads.to_words((spread * rng.standard_normal((n, h, 128))).astype(np.float32), act)
         for k, h in (("q", hq), ("k", hkv), ("v", hkv))}
    elem = np.uint8 if dtype == "e5m2" else np.uint16
    pool = rng.integers(0, np.iinfo(elem).max + 1, size=(nb + 1, 2, hkv, 16, 128), dtype=elem)   # the last: canary
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a).view(np.int16 if a.dtype == np.uint16 else a.dtype)).cuda()  # noqa: E731
    t = _torch_dtype(torch, dtype)
    if packed:   # rows of one projection, with four values to spare between rows
        row = torch.zeros((n, (hq + 2 * hkv) * 128 + 8), dtype=torch.int16, device="cuda")
        flat = dev(np.concatenate([x["q"], x["k"], x["v"]], axis=1).reshape(n, -1))
        row[:, :flat.shape[1]] = flat
        heads = row[:, :flat.shape[1]].unflatten(1, (hq + 2 * hkv, 128)).view(t)
        q, k, v = heads[:, :hq], heads[:, hq:hq + hkv], heads[:, hq + hkv:]
    else:
        q, k, v = (dev(x[name]).view(t) for name in "qkv")
    q_out = q if in_place else torch.full((n, hq, 128), float("nan"), dtype=t, device="cuda")
    d_pool = dev(pool)
    turns = torch.from_numpy(ekv.rope_freqs(rot, **rule).view(np.int64)).cuda()
    print(f"rope: n={n} Hq={hq} Hkv={hkv} {dtype} rot={rot} {layout} packed={packed} in_place={in_place} {rule}", flush=True)
    ekv.rope_append(ekv.make_pool(d_pool[:nb], hkv, dtype), ekv.make_rope(turns, rot, layout, magnitude),
                    dev(positions.astype(np.int32)), dev(slots), q, k, v, q_out, stream)
    torch.cuda.synchronize()
    qf, kf = _values(x["q"], act), _values(x["k"], act)
    mag = float(np.float32(magnitude))
    want_q, want_k = (serve.rotate(a, positions, theta, layout, mag) for a in (qf, kf))
    got_q = _values(q_out.contiguous().view(torch.int16).cpu().numpy().view(np.uint16), act)
    _check(got_q[..., :rot], want_q[..., :rot], _pair_size(qf, rot, layout, mag)[..., :rot], act)
    assert np.array_equal(got_q[..., rot:], qf[..., rot:])
    got = d_pool.cpu().numpy().view(elem)
    in_pool = (slots >= 0) & (slots < nb * 16)
    blk, off = slots[in_pool] // 16, slots[in_pool] % 16
    got_k, got_v = got[blk, 0, :, off], got[blk, 1, :, off]
    _check(_values(got_k, dtype)[..., :rot], want_k[in_pool][..., :rot], _pair_size(kf, rot, layout, mag)[in_pool][..., :rot], dtype)
    # what passes through, and the values: the words themselves, or their nearest E5M2 bytes
    through = lambda w: workloads.f32_to_e5m2_bytes(_values(w, act).astype(np.float32)) if dtype == "e5m2" else w  # noqa: E731
    assert np.array_equal(got_k[..., rot:], through(x["k"][in_pool][..., rot:]))
    assert np.array_equal(got_v, through(x["v"][in_pool]))
    rest = pool.copy()
    rest[blk, 0, :, off], rest[blk, 1, :, off] = got_k, got_v
    assert np.array_equal(got, rest), "a row that no token owns was written"
    if packed and not in_place:
        assert np.array_equal(row.cpu().numpy()[:, :flat.shape[1]], flat.cpu().numpy())
    return got_q


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "e5m2"])
@pytest.mark.parametrize("layout", ["half", "pairs"])
@pytest.mark.parametrize("rot", [16, 48, 64, 112, 128])
def test_types_layouts_and_parts_of_the_head(dtype, layout, rot):
    _run(37, 8, 2, dtype=dtype, layout=layout, rot=rot, magnitude=1.125, seed=rot)


@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 2047, 2048, 2051])
def test_numbers_of_tokens(n):
    _run(n, 4, 2, seed=n, packed=bool(n % 2))


@pytest.mark.parametrize("hq,hkv", [(1, 1), (3, 1), (16, 1), (16, 16), (64, 8), (40, 5), (7, 3)])
@pytest.mark.parametrize("n", [5, 2100])
def test_head_counts(hq, hkv, n):
    _run(n, hq, hkv, seed=hq, dtype="fp16" if hkv % 2 else "bf16")


@pytest.mark.parametrize("rule", [dict(base=500000.0), dict(base=10000.0, scaling="linear", factor=4.0),
                                  dict(base=10000.0, scaling="base", factor=32.0), dict(base=1.0),
                                  dict(base=500000.0, scaling="parts", factor=8.0, context=8192.0, low=1.0, high=4.0)])
@pytest.mark.parametrize("layout", ["half", "pairs"])
def test_frequency_rules_at_far_positions(rule, layout):
    far = [0, 1, 2, 8191, 131071, 1000000, 16777217, 123456789, 2**31 - 1, -1, -77777, -2**31]
    _run(12, 8, 2, rule=rule, layout=layout, positions=far, seed=9)


@pytest.mark.parametrize("dtype", ["bf16", "e5m2"])
@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("n", [33, 3000])
def test_in_place_and_packed_rows(dtype, packed, n):
    _run(n, 8, 4, dtype=dtype, packed=packed, in_place=True, layout="pairs" if packed else "half", rot=96, seed=21)


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "e5m2"])
@pytest.mark.parametrize("n,packed,in_place", [(2047, False, False), (2048, False, True), (2050, True, True)])
def test_inputs_around_32_megabytes(dtype, n, packed, in_place):
    """64 rows of 256 bytes a token: from 2048 tokens on the inputs are read past the caches."""
    _run(n, 40, 12, dtype=dtype, packed=packed, in_place=in_place, layout="pairs" if packed else "half", seed=n)


def test_slots_outside_the_pool_leave_it_as_it_is():
    _run(20, 4, 2, seed=3, skip=[(0, -1), (7, -2**31), (11, 16 * 5), (12, 16 * 5 + 15), (19, 2**31 - 1)], nb=5)


@pytest.mark.parametrize("spread", [1e-6, 3e4])
@pytest.mark.parametrize("dtype", ["fp16", "e5m2"])
def test_small_and_large_values(dtype, spread):
    """fp16 and E5M2 subnormals, and values up to where a turn may overflow to infinity
    (those are left out: |x| + |y| stays below the largest value)."""
    _run(40, 4, 2, dtype=dtype, spread=min(spread, 5000.0), seed=4)


def test_infinities_and_nans_stay_in_their_pairs():
    """A NaN or infinity in one pair reaches that pair alone."""
    torch = require_gpu()
    x = torch.randn((2, 2, 128), device="cuda").bfloat16()
    q = x.clone()
    q[0, 0, 3], q[1, 1, 70] = float("nan"), float("inf")
    kv = torch.zeros((2, 2, 2, 16, 128), dtype=torch.bfloat16, device="cuda")
    turns = torch.from_numpy(ekv.rope_freqs(128).view(np.int64)).cuda()
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    out, clean = torch.empty_like(x), torch.empty_like(x)
    for a, o in ((q, out), (x, clean)):
        ekv.rope_append(ekv.make_pool(kv, 2), ekv.make_rope(turns, 128), i32(7, 9), i32(3, 17), a, a, a, o)
    torch.cuda.synchronize()
    same = torch.ones_like(out, dtype=torch.bool)
    for r, h, i in ((0, 0, 3), (1, 1, 6)):
        same[r, h, i] = same[r, h, i + 64] = False
        assert not torch.isfinite(out[r, h, i]) and not torch.isfinite(out[r, h, i + 64])
    assert torch.equal(out[same], clean[same])


def test_e5m2_rounding_of_every_fp16_value():
    """Values pass to an 8-bit pool through one rounding to nearest even: every finite
    fp16 word, and the infinities, against torch's conversion."""
    torch = require_gpu()
    words = np.arange(1 << 16, dtype=np.uint16)
    words = words[(words & 0x7C00) != 0x7C00]
    words = np.concatenate([words, np.array([0x7C00, 0xFC00], dtype=np.uint16)])
    words = np.concatenate([words, np.zeros(-len(words) % 256, dtype=np.uint16)]).reshape(-1, 2, 128)
    n = len(words)
    v = torch.from_numpy(words.view(np.int16)).cuda().view(torch.float16)
    kv = torch.zeros((n // 16 + 1, 2, 2, 16, 128), dtype=torch.uint8, device="cuda")
    turns = torch.from_numpy(ekv.rope_freqs(16).view(np.int64)).cuda()
    slots = torch.arange(n, dtype=torch.int32, device="cuda")
    ekv.rope_append(ekv.make_pool(kv, 2, "e5m2"), ekv.make_rope(turns, 16), slots, slots, v, v, v, torch.empty_like(v))
    torch.cuda.synchronize()
    got = kv[slots.long() // 16, 1, :, slots.long() % 16].cpu().numpy()
    want = torch.from_numpy(words.view(np.int16)).view(torch.float16).to(torch.float8_e5m2).view(torch.uint8).numpy()
    assert np.array_equal(got, want)


def test_another_stream_and_a_graph():
    torch = require_gpu()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    _run(50, 8, 2, seed=6, stream=side)
    n, hq, hkv = 9, 8, 2
    q, k, v = (torch.randn((n, h, 128), device="cuda").bfloat16() for h in (hq, hkv, hkv))
    kv = torch.zeros((4, 2, hkv, 16, 128), dtype=torch.bfloat16, device="cuda")
    out, pos = torch.empty_like(q), torch.arange(n, dtype=torch.int32, device="cuda")
    slots = torch.arange(5, 5 + n, dtype=torch.int32, device="cuda")
    turns = torch.from_numpy(ekv.rope_freqs(128).view(np.int64)).cuda()
    pool, rope = ekv.make_pool(kv, hkv), ekv.make_rope(turns, 128)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ekv.rope_append(pool, rope, pos, slots, q, k, v, out)
    for replay in range(4):
        q.copy_(torch.randn_like(q)), k.copy_(torch.randn_like(k))
        pos += 1000
        slots += 7
        graph.replay()
        torch.cuda.synchronize()
        got, got_kv = out.clone(), kv.clone()
        out.fill_(0), kv.view(torch.int16)[slots.long() // 16, :, :, slots.long() % 16].fill_(0)
        ekv.rope_append(pool, rope, pos, slots, q, k, v, out)
        torch.cuda.synchronize()
        assert torch.equal(got, out) and torch.equal(got_kv, kv)


def test_append_after_rope_of_position_zero_is_the_plain_append():
    """At position 0 nothing turns: the pool is that of ekv_append_kv."""
    torch = require_gpu()
    rng = np.random.default_rng(8)
    k, v = (rng.integers(0, 0x7F80, size=(6, 2, 128)).astype(np.uint16) for _ in range(2))
    pool = np.zeros((3, 2, 2, 16, 128), dtype=np.uint16)
    slots = np.array([1, 47, 16, 3, 30, 9], dtype=np.int32)
    dev = lambda a: torch.from_numpy(a.view(np.int16) if a.dtype == np.uint16 else a).cuda()  # noqa: E731
    d = dev(pool)
    kd, vd = dev(k).view(torch.bfloat16), dev(v).view(torch.bfloat16)
    turns = torch.from_numpy(ekv.rope_freqs(64).view(np.int64)).cuda()
    ekv.rope_append(ekv.make_pool(d, 2), ekv.make_rope(turns, 64), dev(np.zeros(6, dtype=np.int32)), dev(slots), kd, kd, vd,
                    torch.empty_like(kd))
    torch.cuda.synchronize()
    assert np.array_equal(d.cpu().numpy().view(np.uint16), otr.append(pool, slots, k, v))
