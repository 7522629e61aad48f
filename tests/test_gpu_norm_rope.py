"""Norms of heads, rotation and append on the GPU against the oracle in 64 bits.

Tolerance, in half units u = 2^-24 of 32 bits.  The sum of squares is at most 12
additions deep (12 u, halved by the root), its mean and eps one rounding more (u / 2),
the reciprocal root 2 u, weight + offset, its product with the root and that with the
element u each: below 12 u together, under 2^-20 of a levelled element.  Turning adds
2^-20 (|x| + |y|) of the levelled pair (tests/test_gpu_rope.py), so 2^-19 of it in
all; the one rounding to the output adds half a step of the value, or half the
smallest subnormal."""

import numpy as np
import pytest

from oracle import long_context as olc
from oracle import serve
from paper_2609_33536_amd import ekv, workloads
from tests.gpu_util import require_gpu

pytestmark = pytest.mark.gpu
HALF_STEP = {"bf16": (2.0 ** -8, 2.0 ** -134), "fp16": (2.0 ** -11, 2.0 ** -25), "e5m2": (2.0 ** -3, 2.0 ** -17)}


def _check(got, want, size, dtype):
    """size: |x| + |y| of each element's levelled pair"""
    rel, sub = HALF_STEP[dtype]
    bound = 2.0 ** -19 * size + rel * (np.abs(want) + 2.0 ** -19 * size) + sub
    off = np.abs(got - want)
    bad = ~(off <= bound)
    assert not bad.any(), (f"{bad.sum()} off; worst {np.max(off / np.maximum(bound, 1e-300)):.3f} of the bound; "
                           f"first at {np.argwhere(bad)[0]}: {got[bad][0]} for {want[bad][0]}")


def _pair_size(x, rot, layout, magnitude):
    a = np.abs(x)
    first = np.arange(rot // 2) if layout == "half" else 2 * np.arange(rot // 2)
    second = first + (rot // 2 if layout == "half" else 1)
    out = a.copy()
    out[..., first] = out[..., second] = abs(magnitude) * (a[..., first] + a[..., second])
    return out


def _run(n, hq, hkv, *, dtype="bf16", rot=128, layout="half", magnitude=1.0, weights=("shared", "shared"), offset=0.0,
         eps=1e-6, packed=False, in_place=False, seed=0, skip=(), spread=1.0, stream=None):
    torch = require_gpu()
    rng = np.random.default_rng(seed)
    act = workloads.query_dtype(dtype)
    theta = serve.frequencies(rot, 10000.0)
    positions = rng.integers(0, 1 << 20, size=n)
    nb = n // 16 + 4
    slots = rng.permutation(nb * 16)[:n].astype(np.int32)
    for i, value in skip:
        slots[i] = value
    x = {k: workloads.to_words((spread * rng.uniform(0.1, 3.0, size=(n, h, 1)) * rng.standard_normal((n, h, 128))).astype(np.float32), act)
         for k, h in (("q", hq), ("k", hkv), ("v", hkv))}
    w = {}
    for name, kind, heads in (("q", weights[0], hq), ("k", weights[1], hkv)):
        shape = {"none": None, "shared": (128,), "heads": (heads, 128)}[kind]
        w[name] = None if shape is None else workloads.to_words((1.0 - offset + 0.3 * rng.standard_normal(shape)).astype(np.float32), act)
    elem = np.uint8 if dtype == "e5m2" else np.uint16
    pool = rng.integers(0, np.iinfo(elem).max + 1, size=(nb + 1, 2, hkv, 16, 128), dtype=elem)   # the last: canary
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a).view(np.int16 if a.dtype == np.uint16 else a.dtype)).cuda()  # noqa: E731
    t = torch.bfloat16 if act == "bf16" else torch.float16
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
    d_w = [None if w[i] is None else dev(w[i]).view(t) for i in "qk"]
    turns = torch.from_numpy(ekv.rope_freqs(rot, 10000.0).view(np.int64)).cuda()
    print(f"norm: n={n} Hq={hq} Hkv={hkv} {dtype} rot={rot} {layout} {weights} offset={offset} packed={packed} in_place={in_place}",
          flush=True)
    ekv.norm_rope_append(ekv.make_pool(d_pool[:nb], hkv, dtype), ekv.make_rope(turns, rot, layout, magnitude),
                         ekv.make_head_norm(*d_w, eps, offset), dev(positions.astype(np.int32)), dev(slots), q, k, v, q_out, stream)
    torch.cuda.synchronize()
    mag, eps, offset = float(np.float32(magnitude)), float(np.float32(eps)), float(np.float32(offset))
    level = {i: olc.level(olc.values(x[i], act), None if w[i] is None else olc.values(w[i], act), eps, offset) for i in "qk"}
    turned = {i: serve.rotate(level[i], positions, theta, layout, mag) for i in "qk"}
    for i in "qk":
        turned[i][..., rot:] = level[i][..., rot:]
    got_q = olc.values(q_out.contiguous().view(torch.int16).cpu().numpy().view(np.uint16), act)
    _check(got_q, turned["q"], _pair_size(level["q"], rot, layout, mag), act)
    got = d_pool.cpu().numpy().view(elem)
    live = (slots >= 0) & (slots < nb * 16)
    blk, off = slots[live] // 16, slots[live] % 16
    got_k, got_v = got[blk, 0, :, off], got[blk, 1, :, off]
    _check(olc.values(got_k, dtype), turned["k"][live], _pair_size(level["k"], rot, layout, mag)[live], dtype)
    v_words = x["v"][live]
    if dtype == "e5m2":
        v_words = workloads.f32_to_e5m2_bytes(olc.values(v_words, act).astype(np.float32))
    assert np.array_equal(got_v, v_words)
    rest = pool.copy()
    rest[blk, 0, :, off], rest[blk, 1, :, off] = got_k, got_v
    assert np.array_equal(got, rest), "a row that no token owns was written"
    return got_q


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "e5m2"])
@pytest.mark.parametrize("layout", ["half", "pairs"])
@pytest.mark.parametrize("rot", [16, 48, 64, 112, 128])
def test_types_layouts_and_parts_of_the_head(dtype, layout, rot):
    _run(37, 8, 2, dtype=dtype, layout=layout, rot=rot, magnitude=1.125, seed=rot)


@pytest.mark.parametrize("weights", [(a, b) for a in ("none", "shared", "heads") for b in ("none", "shared", "heads")])
@pytest.mark.parametrize("offset", [0.0, 1.0, -0.25])
def test_weights_of_all_heads_of_each_and_none(weights, offset):
    _run(21, 6, 3, weights=weights, offset=offset, seed=5, dtype="fp16" if offset else "bf16", layout="pairs", rot=64)


@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 700, 2047, 2051])
def test_numbers_of_tokens(n):
    _run(n, 4, 2, seed=n, packed=bool(n % 2), weights=("heads", "shared"))


@pytest.mark.parametrize("hq,hkv", [(1, 1), (3, 1), (16, 1), (16, 16), (64, 8), (40, 5), (7, 3)])
@pytest.mark.parametrize("n", [5, 2100])
def test_head_counts(hq, hkv, n):
    _run(n, hq, hkv, seed=hq, weights=("shared", "heads"), dtype="fp16" if hkv % 2 else "bf16")


@pytest.mark.parametrize("dtype", ["bf16", "e5m2"])
@pytest.mark.parametrize("n,packed,in_place", [(2047, False, False), (2048, False, True), (2050, True, True)])
def test_inputs_around_32_megabytes(dtype, n, packed, in_place):
    """64 rows of 256 bytes a token: from 2048 tokens on the inputs are read past the caches."""
    _run(n, 40, 12, dtype=dtype, packed=packed, in_place=in_place, seed=n)


def test_slots_outside_the_pool_leave_it_as_it_is():
    _run(20, 4, 2, seed=3, skip=[(0, -1), (7, -2**31), (11, 16 * 5), (12, 16 * 5 + 15), (19, 2**31 - 1)])


@pytest.mark.parametrize("eps", [1e-30, 1e-12, 1e-5, 0.5, 1e6])
@pytest.mark.parametrize("spread", [1e-6, 1.0, 1e4])
def test_eps_beside_small_and_large_heads(eps, spread):
    _run(9, 4, 2, eps=eps, spread=spread, seed=11)


@pytest.mark.parametrize("spread", [1e17, 1e18, 3e19, 1e37])
def test_heads_whose_squares_overflow(spread):
    _run(9, 4, 2, spread=spread, seed=12)


def test_zero_heads_stay_zero_and_bad_values_stay_in_their_head():
    torch = require_gpu()
    x = torch.randn((3, 2, 128), device="cuda").bfloat16()
    x[0, 1] = 0.0
    bad = x.clone()
    bad[1, 0, 5], bad[2, 1, 90] = float("nan"), float("inf")
    kv = torch.zeros((2, 2, 2, 16, 128), dtype=torch.bfloat16, device="cuda")
    turns = torch.from_numpy(ekv.rope_freqs(128).view(np.int64)).cuda()
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    out, clean = torch.empty_like(x), torch.empty_like(x)
    for a, o in ((bad, out), (x, clean)):
        ekv.norm_rope_append(ekv.make_pool(kv, 2), ekv.make_rope(turns, 128), ekv.make_head_norm(), i32(7, 9, 1), i32(3, 17, 5), a, a, a, o)
    torch.cuda.synchronize()
    assert (out[0, 1] == 0).all()
    same = torch.ones((3, 2), dtype=torch.bool, device="cuda")
    same[1, 0] = same[2, 1] = False
    assert torch.equal(out[same], clean[same]) and not torch.isfinite(out[1, 0]).any()
    assert torch.isnan(out[2, 1, [26, 90]]).all()


def test_without_weights_a_levelled_head_passes_unchanged():
    """Heads of +-1 have a mean square of exactly 1: with eps far below a step of 1 they
    are the rotation's inputs themselves, up to the reciprocal root's last place."""
    torch = require_gpu()
    q = (torch.randint(0, 2, (5, 4, 128), device="cuda") * 2 - 1).bfloat16()
    kv = [torch.zeros((2, 2, 4, 16, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    turns = torch.from_numpy(ekv.rope_freqs(128).view(np.int64)).cuda()
    rope, pos = ekv.make_rope(turns, 128), torch.arange(5, dtype=torch.int32, device="cuda")
    a, b = torch.empty_like(q), torch.empty_like(q)
    ekv.rope_append(ekv.make_pool(kv[0], 4), rope, pos, pos, q, q, q, a)
    ekv.norm_rope_append(ekv.make_pool(kv[1], 4), rope, ekv.make_head_norm(eps=1e-12), pos, pos, q, q, q, b)
    torch.cuda.synchronize()
    assert (a.float() - b.float()).abs().max() <= 2.0 ** -7 * 2
    assert torch.equal(kv[0][:, 1], kv[1][:, 1])


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
    w = torch.randn(128, device="cuda").bfloat16()
    norm = ekv.make_head_norm(w, w.clone())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ekv.norm_rope_append(pool, rope, norm, pos, slots, q, k, v, out)
    for replay in range(4):
        q.copy_(torch.randn_like(q)), k.copy_(torch.randn_like(k)), w.copy_(torch.randn_like(w))
        pos += 1000
        slots += 7
        graph.replay()
        torch.cuda.synchronize()
        got, got_kv = out.clone(), kv.clone()
        out.fill_(0), kv.view(torch.int16)[slots.long() // 16, :, :, slots.long() % 16].fill_(0)
        ekv.norm_rope_append(pool, rope, norm, pos, slots, q, k, v, out)
        torch.cuda.synchronize()
        assert torch.equal(got, out) and torch.equal(got_kv, kv)
