"""The serving step around the cache: table extension, rotary positions and
decode over shared prefixes (oracle).

TEST INFRASTRUCTURE ONLY (see the package docstring).

The paper's runtime sits in a paged serving engine (§2.1, §3.4); these are
that engine's operators next to the attention, from their definitions:

* ``extend``        -- every sequence in order takes, from the head of a free
  ring, the blocks that its new tokens need; one slot and one position per
  token; everything or nothing.
* ``frequencies``   -- radians a position of each rotated pair.
* ``rotate``        -- pair (x, y) at position t becomes the complex number
  magnitude (x + iy) e^{i t theta}; angles in extended precision, since a far
  position times theta needs more than a double leaves after the turns.
* ``decode_shared`` -- softmax attention over the prefix's tokens followed by
  the sequence's own.
"""

import math

import numpy as np

from . import attention, encoding, fp8, paged

ROW, TOKENS, BLOCKS, BASE_TAIL = 1, 2, 4, 8


def extend(ids, head, count, num_blocks, seq_lens, new_lens, block_table, tags, max_tokens, start=None, page=16):
    """Plain loops over sequences and tokens.  Returns a dict of the arrays that
    the call leaves: table, tags, lens, cu, slots, positions, cursor, status."""
    bt, tags = np.array(block_table, copy=True), np.array(tags, copy=True)
    lens = np.array(seq_lens, dtype=np.int32, copy=True)
    cap = len(ids)
    head, count = int(head) % cap, min(max(int(count), 0), cap)
    reasons, tokens, blocks = 0, 0, 0
    for s, (length, n) in enumerate(zip(seq_lens, new_lens)):
        length, n = int(length), int(n)
        if length < 0 or n < 0 or length + n > bt.shape[1] * page:
            reasons |= ROW
            continue
        tokens += n
        blocks += -(-(length + n) // page) - -(-length // page)
        if n > 0 and length % page and tags[s, length // page]:
            reasons |= BASE_TAIL
    if tokens > max_tokens:
        reasons |= TOKENS
    if blocks > count:
        reasons |= BLOCKS
    cu = np.zeros(len(lens) + 1, dtype=np.int32)
    slots = np.full(max_tokens, -1, dtype=np.int32)
    positions = np.zeros(max_tokens, dtype=np.int32)
    full = 1 << 30
    if reasons:
        return dict(table=bt, tags=tags, lens=lens, cu=cu, slots=slots, positions=positions, cursor=(head, count),
                    status=(reasons, min(tokens, full), min(blocks, full), count))
    row = taken = 0
    for s, (length, n) in enumerate(zip(seq_lens, new_lens)):
        for p in range(int(length), int(length) + int(n)):
            if p % page == 0:
                bt[s, p // page] = ids[(head + taken) % cap]
                tags[s, p // page] = 0
                taken += 1
            block = int(bt[s, p // page])
            slots[row] = block * page + p % page if 0 <= block < num_blocks else -1
            positions[row] = p + (0 if start is None else int(start[s]))
            row += 1
        lens[s] += n
        cu[s + 1] = row
    return dict(table=bt, tags=tags, lens=lens, cu=cu, slots=slots, positions=positions,
                cursor=((head + taken) % cap, count - taken), status=(0, tokens, taken, count - taken))


def frequencies(rotary_dim, base, scaling="none", factor=1.0, context=0.0, low=1.0, high=4.0):
    """theta [rotary_dim / 2] in extended precision."""
    ld = np.longdouble
    i = np.arange(rotary_dim // 2, dtype=ld)
    base, factor = ld(base), ld(factor)
    if scaling == "base":
        base = base * factor ** (ld(rotary_dim) / (rotary_dim - 2))
    theta = base ** (-2 * i / rotary_dim)
    if scaling == "linear":
        theta = theta / factor
    if scaling == "parts":
        turns = ld(context) * theta / (2 * _PI)
        g = np.clip((turns - low) / (ld(high) - low), 0, 1)
        theta = g * theta + (1 - g) * theta / factor
    return theta


_PI = np.longdouble("3.14159265358979323846264338327950288")


def rotate(x, positions, theta, layout, magnitude=1.0):
    """x float64 [n][heads][d], positions int [n], theta [rot / 2]: float64 [n][heads][d]."""
    x = np.asarray(x, dtype=np.float64)
    rot = 2 * len(theta)
    turns = np.asarray(positions, dtype=np.longdouble)[:, None] * theta / (2 * _PI)
    angle = (2 * _PI * (turns - np.rint(turns))).astype(np.float64)
    e = magnitude * np.exp(1j * angle)[:, None, :]
    first = np.arange(rot // 2) if layout == "half" else 2 * np.arange(rot // 2)
    second = first + (rot // 2 if layout == "half" else 1)
    z = (x[..., first] + 1j * x[..., second]) * e
    out = x.copy()
    out[..., first], out[..., second] = z.real, z.imag
    return out


def _gather(pool, bt_row, tag_row, length, dtype):
    if dtype == "e5m2":
        return fp8.gather_sequence(pool, bt_row, tag_row, length)
    return paged.gather_sequence(pool, bt_row, tag_row, length, dtype)


def decode_shared(q, pool, prefix_table, prefix_tags, prefix_lens, group_start, block_table, tags, seq_lens, dtype="bf16",
                  scale=None):
    """q: uint16 [B][Hq][d] words (fp16 for an e5m2 pool).  Returns float64 [B][Hq][d]."""
    bsz, hq, d = q.shape
    group = hq // pool.shape[2]
    scale = 1.0 / math.sqrt(d) if scale is None else scale
    qf = encoding.words_to_f64(np.asarray(q, dtype=np.uint16), "fp16" if dtype == "e5m2" else dtype)
    out = np.zeros((bsz, hq, d))
    parts = {}
    for s in range(bsz):
        p = next((p for p in range(len(prefix_lens)) if group_start[p] <= s < group_start[p + 1]), None)
        k, v = _gather(pool, block_table[s], tags[s], int(seq_lens[s]), dtype)
        if p is not None:
            if p not in parts:
                parts = {p: _gather(pool, prefix_table[p], prefix_tags[p], int(prefix_lens[p]), dtype)}
            k, v = np.concatenate([parts[p][0], k]), np.concatenate([parts[p][1], v])
        if len(k) == 0:
            continue
        for h in range(hq):
            scores = scale * (k[:, h // group] @ qf[s, h])
            out[s, h] = attention._softmax_weighted(scores, v[:, h // group])
    return out
