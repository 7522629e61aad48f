"""Performance cases of the operators of a long-context decode step over the paged KV cache.

Four operators that a layer of such a step runs one after the other:

* norm: each query and key head divided by its root mean square and weighted, then turned by its position, the keys
  and the values written to their cache slots;
* bounds: the smallest and the largest executed key of each channel of a block, for the blocks that new tokens changed;
* select: for each sequence and KV head the blocks whose bounds allow the largest scores against its queries, next to
  its first and its newest blocks;
* attend: decode attention over the selected blocks alone.

With ``own`` false, ``run`` computes them in their plain form (elementary torch operations in 32 bits; the scores of
the selection, which decide between close neighbours, in 64); with ``own`` true it makes the calls that a user makes of
the package.  Shapes are the package's own workloads (Llama-3.1-8B: 32 query / 8 KV heads, 70B: 64 / 8, head dim 128,
pages of 16 tokens) or generic sizes around them.
"""

import math

import numpy as np
import torch

own = False

D, PAGE = 128, 16
SCALE = 1.0 / math.sqrt(D)


def listed():
    norm = dict(kind="norm", base=500000.0, layout="half", rot=128, weights="shared", offset=0.0, eps=1e-6, packed=True)
    bounds = dict(kind="bounds", placement="random", base=0.0)
    select = dict(kind="select", sink=1)
    attend = dict(kind="attend", sink=1, recent=4, placement="random")
    return [
        # The newest token of each of 64 sequences of the 8B layer: a launch.
        dict(norm, name="norm-decode", n=64, hq=32, hkv=8, dtype="bf16", far=131072, span=1),
        # An odd number of tokens, weights of their own for each head (stored less one), a quarter of the head turned.
        dict(norm, name="norm-heads", n=1337, hq=16, hkv=16, dtype="fp16", layout="pairs", rot=32, base=10000.0,
             weights="heads", offset=1.0, eps=1e-5, far=1000000, span=191, packed=False),
        # A long prompt with the 70B heads over an 8-bit pool: the largest.
        dict(norm, name="norm-70b-e5m2", n=16384, hq=64, hkv=8, dtype="e5m2", far=65536, span=4096),
        # One decode step of 64 sequences of the 8B layer: the block of each one's newest token.
        dict(bounds, name="bounds-decode", batch=64, hq=32, hkv=8, dtype="bf16", len_lo=2048, len_hi=8192, new_lo=1, new_hi=1),
        # 16 ragged prompts of the 8B layer after their prefill, all of their blocks.
        dict(bounds, name="bounds-prompts", batch=16, hq=32, hkv=8, dtype="bf16", len_lo=4097, len_hi=16384, new_lo=16384,
             new_hi=16384),
        # An 8-bit pool of the 70B heads after a round of transitions, the older half now 4-bit BASE: all anew; the largest.
        dict(bounds, name="bounds-70b-e5m2", batch=48, hq=64, hkv=8, dtype="e5m2", len_lo=8192, len_hi=16384, new_lo=16384,
             new_hi=16384, base=0.5, placement="oldest"),
        # A few short requests, fewer blocks than the budget for some: all latency.
        dict(select, name="select-tiny", batch=4, hq=8, hkv=2, dtype="bf16", len_lo=100, len_hi=1000, budget=32, recent=2),
        # The 8B layer over long ragged contexts, one in 12 blocks of them.
        dict(select, name="select-8b", batch=32, hq=32, hkv=8, dtype="bf16", len_lo=16384, len_hi=32768, budget=128, recent=4),
        # One reader of a million tokens, 70B heads: few rows, each very long.
        dict(select, name="select-million", batch=1, hq=64, hkv=8, dtype="fp16", len_lo=1000001, len_hi=1000001, budget=256,
             recent=4),
        # One sequence at the same budget: few rows, the smallest.
        dict(attend, name="attend-one", batch=1, hq=64, hkv=8, dtype="fp16", len_lo=20001, len_hi=20001, budget=256, base=0.0),
        # The 8B decode layer at full batch: 2048 of up to 16384 tokens, a quarter of the cache BASE.
        dict(attend, name="attend-8b", batch=64, hq=32, hkv=8, dtype="bf16", len_lo=4096, len_hi=16384, budget=128, base=0.25),
        # The 70B heads over an 8-bit pool, 8192 of up to 32768 tokens, the older half 4-bit BASE; the largest.
        dict(attend, name="attend-70b-e5m2", batch=48, hq=64, hkv=8, dtype="e5m2", len_lo=16384, len_hi=32768, budget=512,
             base=0.5, placement="oldest"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm", "bounds", "select", "select", "attend", "attend"])
    hq, hkv = rng.choice([(8, 2), (32, 8), (32, 8), (32, 8), (64, 8), (64, 8), (32, 4), (16, 16), (16, 8), (16, 1)])
    dtype = rng.choice(["bf16", "bf16", "fp16", "e5m2"])
    if kind == "norm":
        n = _log(rng, 1, 15360)
        return dict(kind=kind, n=n, hq=hq, hkv=hkv, dtype=dtype, layout=rng.choice(["half", "pairs"]),
                    rot=rng.choice([128, 128, 64, 96, 32, 16]), base=rng.choice([10000.0, 500000.0]),
                    weights=rng.choice(["none", "shared", "shared", "heads"]), offset=rng.choice([0.0, 0.0, 1.0]),
                    eps=rng.choice([1e-6, 1e-5]), far=_log(rng, 64, 1000000), span=_log(rng, 1, n), packed=rng.random() < 0.5)
    base, placement = rng.choice([0.0, 0.0, 0.5, 1.0, rng.uniform(0.05, 0.95)]), rng.choice(["random", "oldest"])
    batch, length, spread = _log(rng, 1, 256), _log(rng, 1, 131072), rng.uniform(1.0, 4.0)
    if kind == "bounds":
        while batch * length * hkv > 16 * 16384 * 8:
            batch, length = max(1, batch * 3 // 4), max(1, length * 3 // 4)
        new = rng.choice([1, length, _log(rng, 1, length)])
        return dict(kind=kind, batch=batch, hq=hq, hkv=hkv, dtype=dtype, len_lo=max(1, int(length / spread)), len_hi=length,
                    new_lo=rng.choice([0, new]), new_hi=new, base=base, placement=placement)
    sink, recent = rng.choice([0, 1, 1, 2, 4]), rng.choice([1, 1, 2, 4, 8])
    if kind == "select":
        length = _log(rng, 1, 1000001)
        while batch * length * hkv > 1000001 * 8:
            batch, length = max(1, batch * 3 // 4), max(1, length * 3 // 4)
        budget = max(sink + recent, _log(rng, 1, 1024))
        return dict(kind=kind, batch=batch, hq=hq, hkv=hkv, dtype=dtype, len_lo=max(1, int(length / spread)), len_hi=length,
                    budget=budget, sink=sink, recent=recent)
    budget = _log(rng, 1, 1024)
    # no more tokens attended and no more cache than the largest listed case
    while batch * budget * hkv > 64 * 128 * 8 or batch * length * hkv > 64 * 16384 * 8:
        batch, budget, length = max(1, batch * 3 // 4), max(1, budget * 4 // 5), max(1, length * 3 // 4)
    budget = max(sink + recent, budget)
    return dict(kind=kind, batch=batch, hq=hq, hkv=hkv, dtype=dtype, len_lo=max(1, int(length / spread)), len_hi=length,
                budget=budget, sink=sink, recent=recent, base=base, placement=placement)


# ---- shapes, fixed by the case alone ------------------------------------------

def _whole(lo, hi, n, salt):
    return np.random.default_rng(1000003 * lo + 101 * hi + 7 * n + salt).integers(lo, hi + 1, size=n).astype(np.int32)


def _lengths(case):
    return _whole(case["len_lo"], case["len_hi"], case["batch"], 1)


def _known(case):
    """Tokens whose bounds are there already."""
    lens = _lengths(case)
    return np.maximum(lens - _whole(case["new_lo"], case["new_hi"], case["batch"], 2), 0).astype(np.int32)


def _blocks(lens):
    return (lens + PAGE - 1) // PAGE


def _base_pairs(case):
    """BASE pairs of each sequence (the pair of the newest token stays TARGET)."""
    return np.floor(case["base"] * ((_lengths(case) - 1) // (2 * PAGE)) + 0.5).astype(np.int64)


def _width(lens):
    n = int(_blocks(lens).max())
    return max(2, n + n % 2)


def _elem(case):
    return 1 if case["dtype"] == "e5m2" else 2


TORCH = {"bf16": torch.bfloat16, "fp16": torch.float16, "e5m2": torch.float8_e5m2}


def _query_type(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float16


def _generators(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return np.random.default_rng(seed), gen


def _cuda(a, dtype=None):
    return torch.from_numpy(np.ascontiguousarray(a if dtype is None else np.asarray(a, dtype=dtype))).cuda()


# ---- inputs -------------------------------------------------------------------

def prepare(case, seed):
    return {"norm": _prepare_norm, "bounds": _prepare_bounds, "select": _prepare_select,
            "attend": _prepare_attend}[case["kind"]](case, seed)


def _prepare_norm(case, seed):
    """New tokens in runs of consecutive positions, each run in its own blocks of a pool with some blocks to spare."""
    rng, gen = _generators(seed)
    n, hq, hkv, span = case["n"], case["hq"], case["hkv"], case["span"]
    runs = -(-n // span)
    first = rng.integers(0, max(1, case["far"] - span), size=runs)
    token = np.arange(n)
    pos = first[token // span] + token % span
    per = -(-(span + PAGE - 1) // PAGE)                       # blocks that a run may touch
    blocks = rng.permutation(runs * per + 5)
    at = first[token // span] % PAGE + token % span            # place of a token in its run's blocks
    slots = blocks[(token // span) * per + at // PAGE] * PAGE + at % PAGE
    act = _query_type(case)
    # (heads of a projection differ in size; the norm is there to level them)
    make = lambda h: (torch.randn((n, h, D), generator=gen, device="cuda")  # noqa: E731
                      * torch.rand((h, 1), generator=gen, device="cuda").add(0.1).mul(4.0)).to(act)
    if case["packed"]:   # as one projection leaves them: query, key and value heads of a token side by side
        qkv = make(hq + 2 * hkv)
        q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
    else:
        q, k, v = make(hq), make(hkv), make(hkv)
    weight = {}
    for name, heads in (("q", hq), ("k", hkv)):
        shape = {"none": None, "shared": (D,), "heads": (heads, D)}[case["weights"]]
        weight[name] = None if shape is None else (
            torch.randn(shape, generator=gen, device="cuda").mul(0.2).add(1.0 - case["offset"]).to(act))
    kv = torch.randn((len(blocks), 2, hkv, PAGE, D), generator=gen, device="cuda").to(TORCH[case["dtype"]])
    theta = case["base"] ** (-2.0 * np.arange(case["rot"] // 2, dtype=np.float64) / case["rot"])
    st = dict(kind="norm", case=case, q=q, k=k, v=v, kv=kv, positions=_cuda(pos, np.int32), slots=_cuda(slots, np.int32),
              q_out=torch.empty((n, hq, D), dtype=act, device="cuda"), theta=_cuda(theta), weight=weight)
    if own:
        from paper_2609_33536_amd import ekv
        st["freqs"] = torch.from_numpy(ekv.rope_freqs(case["rot"], case["base"]).view(np.int64)).cuda()
        st["rope"] = ekv.make_rope(st["freqs"], case["rot"], case["layout"])
        st["norm"] = ekv.make_head_norm(weight["q"], weight["k"], case["eps"], case["offset"])
        st["pool"] = ekv.make_pool(kv, hkv, case["dtype"])
    return st


def _words(t):
    return t.view(torch.uint8) if t.element_size() == 1 else t.view(torch.int16)


def _pack(kv, first, second):
    """BASE pairs: the high halves of both blocks' elements, side by side in the first block."""
    b = kv.view(torch.uint8)
    if kv.element_size() == 2:
        hi = lambda x: b[x].view(*b[x].shape[:-1], D, 2)[..., 1]  # noqa: E731
    else:
        hi = lambda x: (b[x][..., 0::2] >> 4) | (b[x][..., 1::2] & 0xF0)  # noqa: E731
    b[first] = torch.stack([hi(first), hi(second)], dim=3).reshape(b[first].shape)


def _cache(case, rng, gen):
    """A pool with its blocks in random order, some pairs BASE, and the sequences' table and tags."""
    lens, hkv = _lengths(case), case["hkv"]
    used, width, n = _blocks(lens), _width(lens), int(_blocks(lens).sum())
    ids = rng.permutation(n).astype(np.int32)
    edge = np.concatenate([[0], np.cumsum(used)])
    kv = torch.empty((n, 2, hkv, PAGE, D), dtype=TORCH[case["dtype"]], device="cuda")
    centre = torch.randn((hkv, 1, D), generator=gen, device="cuda") * 0.5   # (keys of a head share a mean)
    step = max(1, (1 << 27) // (2 * hkv * PAGE * D))
    for a in range(0, n, step):
        x = torch.randn((min(step, n - a), 2, hkv, PAGE, D), generator=gen, device="cuda")
        x[:, 0] += centre
        kv[a:a + step] = x.to(kv.dtype)
    table, tag, pairs = np.zeros((len(lens), width), dtype=np.int32), np.zeros((len(lens), width), dtype=np.uint8), []
    for s, base in enumerate(_base_pairs(case)):
        table[s, :used[s]] = ids[edge[s]:edge[s + 1]]
        full = int((lens[s] - 1) // (2 * PAGE))
        js = np.arange(base) if case["placement"] == "oldest" else np.sort(rng.permutation(full)[:base])
        pairs.append(np.stack([table[s, 2 * js], table[s, 2 * js + 1]], axis=1))
        table[s, 2 * js + 1] = table[s, 2 * js]
        tag[s, 2 * js] = tag[s, 2 * js + 1] = 1
    pairs = np.concatenate(pairs).astype(np.int64)
    for a in range(0, len(pairs), 4096):
        _pack(kv, _cuda(pairs[a:a + 4096, 0]), _cuda(pairs[a:a + 4096, 1]))
    st = dict(kind=case["kind"], kv=kv, hq=case["hq"], hkv=hkv, lens=_cuda(lens), table=_cuda(table), tags=_cuda(tag),
              base=len(pairs) > 0)
    if own:
        from paper_2609_33536_amd import ekv
        st["pool"] = ekv.make_pool(_words(kv), hkv, case["dtype"])
        st["batch"] = ekv.make_batch(st["lens"], st["table"], st["tags"], None, case["hq"],
                                     ekv.MODE_GENERAL if len(pairs) else ekv.MODE_NATIVE, int(lens.max()))
    return st


def _prepare_bounds(case, seed):
    """A cache whose newest tokens have just been appended, and the bounds as they were before."""
    rng, gen = _generators(seed)
    st = _cache(case, rng, gen)
    shape = (case["batch"], case["hkv"], _width(_lengths(case)), 2, D)
    st["bounds"] = torch.zeros(shape, dtype=torch.int16 if _elem(case) == 2 else torch.uint8, device="cuda").view(st["kv"].dtype)
    known = _known(case)
    st["known"] = _cuda(known)
    first, last = known // PAGE, _blocks(_lengths(case))
    rows = [(s, b) for s in range(case["batch"]) for b in range(first[s], last[s])]
    st["changed"] = _cuda(np.array(rows, dtype=np.int64).reshape(-1, 2))   # (the plain form's plan: sequence, block)
    return st


def _prepare_select(case, seed):
    """Bounds of the blocks of each sequence: channels around a mean of their own, and queries N(0, 1)."""
    rng, gen = _generators(seed)
    lens, hkv, b = _lengths(case), case["hkv"], case["batch"]
    width, kind = _width(lens), TORCH[case["dtype"]]
    bounds = torch.empty((b, hkv, width, 2, D), dtype=kind, device="cuda")
    centre = torch.randn((b, hkv, 1, 1, D), generator=gen, device="cuda") * 0.5
    step = max(1, (1 << 25) // (b * hkv * D))
    for a in range(0, width, step):   # the extremes of 16 normal keys: about 1.77 from the mean, give or take 0.5
        some = min(step, width - a)
        away = torch.randn((b, hkv, some, 2, D), generator=gen, device="cuda").mul_(0.5).add_(1.77).clamp_(min=0.1)
        away[:, :, :, 0].neg_()
        bounds[:, :, a:a + some] = (centre + away).to(kind)
    q = torch.randn((b, case["hq"], D), generator=gen, device="cuda").to(_query_type(case))
    table = torch.arange(b * width, dtype=torch.int32, device="cuda").view(b, width)
    st = dict(kind="select", case=case, bounds=bounds, q=q, lens=_cuda(lens), table=table,
              selected=torch.empty((b, hkv, case["budget"]), dtype=torch.int32, device="cuda"),
              counts=torch.empty((b, hkv), dtype=torch.int32, device="cuda"))
    if own:
        from paper_2609_33536_amd import ekv
        # (the pool that the table names: a selection does not read it)
        st["kv"] = torch.empty(256, dtype=torch.uint8, device="cuda")
        st["pool"] = ekv.Pool(st["kv"].data_ptr(), b * width, hkv, PAGE, D, {"bf16": 0, "fp16": 1, "e5m2": 3}[case["dtype"]])
        st["batch"] = ekv.make_batch(st["lens"], table, None, None, case["hq"], ekv.MODE_NATIVE, int(lens.max()))
        st["ws"] = ekv.select_workspace(st["pool"], st["batch"], case["budget"])
    return st


def _prepare_attend(case, seed):
    """A cache, queries, and for each sequence and KV head its first and newest blocks and others at random."""
    rng, gen = _generators(seed)
    st = _cache(case, rng, gen)
    b, hkv, budget = case["batch"], case["hkv"], case["budget"]
    blocks = _blocks(st["lens"].long())[:, None, None]
    width = max(st["table"].shape[1], budget)
    at = torch.arange(width, device="cuda")
    rank = torch.rand((b, hkv, width), generator=gen, device="cuda")
    rank = torch.where((at < case["sink"]) | (at >= blocks - case["recent"]), 2.0, rank)
    rank = torch.where(at < blocks, rank, -1.0)
    kept = rank.topk(budget, dim=-1).indices
    kept = torch.where(kept < blocks, kept, 1 << 30).sort(dim=-1).values
    st["selected"] = torch.where(kept < (1 << 30), kept, -1).int()
    st["counts"] = (st["selected"] >= 0).sum(-1).int()
    st["q"] = torch.randn((b, case["hq"], D), generator=gen, device="cuda").to(_query_type(case))
    st["out"] = torch.empty_like(st["q"])
    if own:
        from paper_2609_33536_amd import ekv
        st["ws"] = ekv.decode_selected_workspace(st["pool"], st["batch"], budget)
    return st


# ---- one pass -----------------------------------------------------------------

def run(state):
    st = state
    if st["kind"] == "norm":
        if own:
            from paper_2609_33536_amd import ekv
            ekv.norm_rope_append(st["pool"], st["rope"], st["norm"], st["positions"], st["slots"], st["q"], st["k"], st["v"],
                                 st["q_out"])
        else:
            _plain_norm(st)
        return {"q": st["q_out"], "kv": st["kv"]}
    if st["kind"] == "bounds":
        if own:
            from paper_2609_33536_amd import ekv
            ekv.key_bounds(st["pool"], st["batch"], st["bounds"], st["known"])
        else:
            _plain_bounds(st)
        return {"bounds": st["bounds"]}
    if st["kind"] == "select":
        if own:
            from paper_2609_33536_amd import ekv
            ekv.select_blocks(st["pool"], st["batch"], st["q"], st["bounds"], st["selected"], st["counts"], st["ws"],
                              st["case"]["sink"], st["case"]["recent"])
        else:
            _plain_select(st)
        return {"selected": st["selected"], "counts": st["counts"]}
    if own:
        from paper_2609_33536_amd import ekv
        ekv.attn_decode_selected(st["pool"], st["batch"], st["selected"], st["counts"], st["q"], st["out"], SCALE, st["ws"])
    else:
        _plain_attend(st)
    return {"out": st["out"]}


def _plain_norm(st):
    case, rot = st["case"], st["case"]["rot"]
    angle = st["positions"].double()[:, None, None] * st["theta"]   # (far positions need 64 bits)
    cos, sin = angle.cos().float(), angle.sin().float()

    def level(x, w):
        x = x.float()
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + case["eps"])
        return x if w is None else x * (w.float() + case["offset"])

    def turn(x):
        y = x.clone()
        if case["layout"] == "half":
            a, b = x[..., :rot // 2], x[..., rot // 2:rot]
            y[..., :rot // 2], y[..., rot // 2:rot] = a * cos - b * sin, b * cos + a * sin
        else:
            a, b = x[..., 0:rot:2], x[..., 1:rot:2]
            y[..., 0:rot:2], y[..., 1:rot:2] = a * cos - b * sin, b * cos + a * sin
        return y

    st["q_out"].copy_(turn(level(st["q"], st["weight"]["q"])))
    kv, slot = st["kv"], st["slots"].long()
    for plane, x in ((0, turn(level(st["k"], st["weight"]["k"]))), (1, st["v"].float())):
        _words(kv)[slot // PAGE, plane, :, slot % PAGE] = _words(x.to(kv.dtype))


def _executed(st, phys, tag, member, plane):
    """The executed values of one plane [...][Hkv][16][D] in 32 bits of the blocks phys [...], where tag is 1 as that
    member of a BASE pair."""
    kv = st["kv"]
    blocks = _words(kv)[phys, plane].view(kv.dtype)
    if not st["base"]:
        return blocks.float()
    b, lead, h = blocks.view(torch.uint8), phys.shape, kv.shape[2]
    second = (member == 1)[..., None, None, None]
    packed = b.reshape(*lead, h, 2, PAGE, -1)
    byte = torch.where(second, packed[..., 1, :, :], packed[..., 0, :, :])
    if kv.element_size() == 2:
        base = (byte.to(torch.int16) << 8).view(kv.dtype)
    else:
        base = torch.stack([byte << 4, byte & 0xF0], dim=-1).reshape(blocks.shape).view(kv.dtype)
    return torch.where(tag[..., None, None, None] == 1, base.float(), blocks.float())


def _plain_bounds(st):
    step = max(1, (1 << 26) // (st["hkv"] * PAGE * D))
    for a in range(0, len(st["changed"]), step):
        s, i = st["changed"][a:a + step].unbind(1)
        x = _executed(st, st["table"][s, i].long(), st["tags"][s, i], i % 2, 0)
        here = (i[:, None] * PAGE + torch.arange(PAGE, device="cuda") < st["lens"][s][:, None])[:, None, :, None]
        low = x.masked_fill(~here, math.inf).amin(2)
        high = x.masked_fill(~here, -math.inf).amax(2)
        _words(st["bounds"])[s, :, i] = _words(torch.stack([low, high], dim=2).to(st["kv"].dtype))


def _plain_select(st):
    case, lens = st["case"], st["lens"].long()
    b, hkv, width = st["bounds"].shape[:3]
    q = st["q"].double().view(b, hkv, -1, D)
    up, down = q.clamp(min=0).sum(2)[:, :, None], q.clamp(max=0).sum(2)[:, :, None]
    score = torch.empty((b, hkv, width), dtype=torch.float64, device="cuda")
    step = max(1, (1 << 24) // (b * hkv * D))
    for a in range(0, width, step):   # (close neighbours need 64 bits)
        x = st["bounds"][:, :, a:a + step].double()
        score[:, :, a:a + step] = (x[..., 1, :] * up + x[..., 0, :] * down).sum(-1)
    at, blocks = torch.arange(width, device="cuda"), _blocks(lens)[:, None, None]
    score = score.masked_fill((at < case["sink"]) | (at >= blocks - case["recent"]), math.inf)
    score = score.masked_fill(at >= blocks, -math.inf)
    order = torch.sort(score, dim=-1, descending=True, stable=True).indices[..., :case["budget"]]
    order = torch.where(order < blocks, order, width).sort(dim=-1).values
    st["selected"].fill_(-1)
    st["selected"][..., :order.shape[-1]] = torch.where(order < width, order, -1).int()
    st["counts"].copy_(blocks[..., 0].clamp(max=case["budget"]).expand(b, hkv))


def _plain_attend(st):
    hq, hkv, b = st["hq"], st["hkv"], len(st["q"])
    q = st["q"].float().view(b, hkv, hq // hkv, D)
    for s0 in range(0, b, 8):
        rows = torch.arange(s0, min(b, s0 + 8), device="cuda")
        kept = st["selected"][rows].long()
        there = kept >= 0
        i = kept.clamp(min=0)
        s = rows[:, None, None]
        phys, tag = st["table"][s, i].long(), st["tags"][s, i]
        head = torch.arange(hkv, device="cuda")[None, :, None]
        part = []
        for plane in (0, 1):
            words = _words(st["kv"])[phys, plane, head].view(st["kv"].dtype)
            raw = words.view(torch.uint8).reshape(*phys.shape, 2, PAGE, -1)
            byte = torch.where((i % 2 == 1)[..., None, None], raw[..., 1, :, :], raw[..., 0, :, :])
            if st["kv"].element_size() == 2:
                base = (byte.to(torch.int16) << 8).view(st["kv"].dtype)
            else:
                base = torch.stack([byte << 4, byte & 0xF0], dim=-1).reshape(words.shape).view(st["kv"].dtype)
            part.append(torch.where(tag[..., None, None] == 1, base.float(), words.float()))
        live = there[..., None] & (i[..., None] * PAGE + torch.arange(PAGE, device="cuda") < st["lens"][rows][:, None, None, None])
        k, v = (x.reshape(len(rows), hkv, -1, D) for x in part)
        live = live.reshape(len(rows), hkv, -1)
        v = v.masked_fill(~live[..., None], 0.0)
        scores = (torch.matmul(q[rows], k.transpose(2, 3).contiguous()) * SCALE).masked_fill(~live[:, :, None], -math.inf)
        weight = (scores - scores.amax(-1, keepdim=True)).exp()
        st["out"][rows] = (torch.matmul(weight, v) / weight.sum(-1, keepdim=True)).view(len(rows), hq, D).to(st["out"].dtype)


# ---- what a pass cannot do without -----------------------------------------------

def work(case):
    """Each input once and each output once; attention: 4 flops per score and channel, rotation: 6 per pair, norm: 4 per
    element, bounds: 2 comparisons per element, selection: 4 flops per block and channel."""
    hq, hkv, elem = case["hq"], case["hkv"], _elem(case)
    if case["kind"] == "norm":
        n = case["n"]
        heads = {"none": 0, "shared": 2, "heads": hq + hkv}[case["weights"]]
        size = n * D * (2 * hq * 2 + 2 * hkv * (2 + elem)) + 8 * n + 8 * case["rot"] // 2 + 2 * D * heads
        return {"bytes": float(size), "flops": n * (hq + hkv) * (6.0 * case["rot"] / 2 + 4.0 * D)}
    lens, b = _lengths(case), case["batch"]
    blocks = _blocks(lens)
    if case["kind"] == "bounds":
        first = _known(case) // PAGE
        rows = int(np.maximum(lens - first * PAGE, 0).sum())
        changed = int(np.maximum(blocks - first, 0).sum())
        base = _base_pairs(case)
        if case["placement"] == "oldest":   # BASE tokens among those read
            halved = int(np.maximum(2 * base - first, 0).sum()) * PAGE
        else:
            halved = float((2 * base / np.maximum(blocks, 1) * np.maximum(blocks - first, 0)).sum()) * PAGE
        return {"bytes": (rows - halved / 2) * hkv * D * elem + changed * (2 * hkv * D * elem + 4) + 8.0 * b,
                "flops": 2.0 * rows * hkv * D}
    budget = case["budget"]
    chosen = int(np.minimum(blocks, budget).sum())
    if case["kind"] == "select":
        return {"bytes": float(int(blocks.sum()) * hkv * 2 * D * elem + b * hq * D * 2 + 4 * b + 4 * b * hkv * (budget + 1)),
                "flops": 4.0 * int(blocks.sum()) * hkv * D}
    share = 2.0 * _base_pairs(case) / np.maximum(blocks, 1)   # (blocks at random: BASE in their share)
    tokens = np.minimum(np.minimum(blocks, budget) * PAGE, lens)
    return {"bytes": float((tokens * (1 - share / 2)).sum()) * 2 * hkv * D * elem + b * hq * D * 4 + 4.0 * (b * hkv + chosen * hkv),
            "flops": 4.0 * hq * D * int(tokens.sum())}


# ---- 64-bit reference --------------------------------------------------------------

def exact(case, seed):
    """The definitions, pair by pair of channels, token by token or head by head, in 64 bits."""
    if case["kind"] == "select":
        return None   # whole numbers only
    st = prepare(case, seed)
    return {"norm": _exact_norm, "bounds": _exact_bounds, "attend": _exact_attend}[case["kind"]](case, st)


def _exact_norm(case, st):
    rot, kv = case["rot"], st["kv"].double()
    done = []
    for name in ("q", "k"):
        x, w = st[name].double(), st["weight"][name]
        square = torch.zeros(x.shape[:2], dtype=torch.float64, device="cuda")
        for i in range(D):
            square += x[..., i] ** 2
        x = x / torch.sqrt(square / D + case["eps"])[..., None]
        if w is not None:
            x = x * (w.double() + case["offset"])
        y = x.clone()
        for i in range(rot // 2):   # pair by pair
            one, two = (i, i + rot // 2) if case["layout"] == "half" else (2 * i, 2 * i + 1)
            phase = (st["positions"].double() * case["base"] ** (-2.0 * i / rot))[:, None]
            y[..., one] = x[..., one] * torch.cos(phase) - x[..., two] * torch.sin(phase)
            y[..., two] = x[..., two] * torch.cos(phase) + x[..., one] * torch.sin(phase)
        done.append(y)
    block, row = st["slots"].long() // PAGE, st["slots"].long() % PAGE
    for plane, x in ((0, done[1]), (1, st["v"].double())):
        # (an 8-bit pool holds the nearest 8-bit values: those are what it stands for)
        kv[block, plane, :, row] = x.to(st["kv"].dtype).double() if case["dtype"] == "e5m2" else x
    return {"q": done[0], "kv": kv}


def _exact_values(st, s, rows, blocks, plane):
    """One plane's executed values [len(blocks)][Hkv][16][D] of sequence s, in 64 bits."""
    words = _words(st["kv"])[rows, plane]
    x = words.view(st["kv"].dtype).double()
    base = torch.nonzero(st["tags"][s, blocks] == 1)[:, 0]
    if len(base):
        raw = words[base].view(torch.uint8).reshape(len(base), st["hkv"], 2, -1)
        half = raw[torch.arange(len(base), device="cuda"), :, blocks[base] % 2].to(torch.int32)
        if st["kv"].element_size() == 2:
            value = (half * 256).to(torch.int16).view(st["kv"].dtype)
        else:
            value = torch.stack([(half % 16) * 16, half - half % 16], dim=-1).to(torch.uint8).view(st["kv"].dtype)
        x[base] = value.double().reshape(len(base), st["hkv"], PAGE, D)
    return x


def _exact_bounds(case, st):
    out = st["bounds"].double()
    first, lens = _known(case) // PAGE, _lengths(case)
    for s in range(case["batch"]):
        n = int(_blocks(lens[s:s + 1])[0])
        if first[s] >= n:
            continue
        at = torch.arange(int(first[s]), n, device="cuda")
        x = _exact_values(st, s, st["table"][s, at].long(), at, 0)
        low, high = x[:, :, 0].clone(), x[:, :, 0].clone()
        for t in range(1, PAGE):
            here = (at * PAGE + t < int(lens[s]))[:, None, None]
            low = torch.where(here & (x[:, :, t] < low), x[:, :, t], low)
            high = torch.where(here & (x[:, :, t] > high), x[:, :, t], high)
        out[s, :, at] = torch.stack([low, high], dim=2).transpose(0, 1)
    return {"bounds": out}


def _exact_attend(case, st):
    group = st["hq"] // st["hkv"]
    out = torch.empty(st["q"].shape, dtype=torch.float64, device="cuda")
    lens, counts = _lengths(case), st["counts"].cpu().numpy()
    for s in range(case["batch"]):
        for h in range(st["hkv"]):
            at = st["selected"][s, h, :int(counts[s, h])].long()
            rows = st["table"][s, at].long()
            words = _words(st["kv"])[rows, :, h]
            x = words.view(st["kv"].dtype).double()
            base = torch.nonzero(st["tags"][s, at] == 1)[:, 0]
            if len(base):
                raw = words[base].view(torch.uint8).reshape(len(base), 2, 2, -1)
                half = raw[torch.arange(len(base), device="cuda"), :, at[base] % 2].to(torch.int32)
                if st["kv"].element_size() == 2:
                    value = (half * 256).to(torch.int16).view(st["kv"].dtype)
                else:
                    value = torch.stack([(half % 16) * 16, half - half % 16], dim=-1).to(torch.uint8).view(st["kv"].dtype)
                x[base] = value.double().reshape(len(base), 2, PAGE, D)
            live = (at[:, None] * PAGE + torch.arange(PAGE, device="cuda") < int(lens[s])).reshape(-1)
            k, v = x[:, 0].reshape(-1, D)[live], x[:, 1].reshape(-1, D)[live]
            q = st["q"][s, h * group:(h + 1) * group].double()
            out[s, h * group:(h + 1) * group] = torch.softmax(q @ k.T / math.sqrt(D), dim=1) @ v
    return {"out": out}
