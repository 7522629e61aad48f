"""The long-context decode step: norms of heads, key bounds, block selection and
decode over selected blocks (oracle).

TEST INFRASTRUCTURE ONLY (see the package docstring).

The operators of a paged serving engine that reads a part of a long context, from
their definitions:

* ``level``   -- each head divided by the root of the mean of its squares plus eps,
  times offset + weight.
* ``bounds``  -- per block, KV head and channel the smallest and largest executed
  key, as words.  Words are ordered as sign and magnitude, so -0 is below 0 and a NaN
  beyond the infinity of its sign.
* ``select``  -- a block's score is the sum over channels of the larger of q lo and
  q hi, over the query heads of a KV head; first and newest blocks, then the largest
  scores, what is no number above infinity, the lowest block first among equals.
* ``decode``  -- softmax attention over the tokens of the listed blocks.
"""

import math

import numpy as np

from . import encoding, fp8, paged


def level(x, weight, eps, offset=0.0):
    """x float64 [n][heads][128]; weight float64 [128], [heads][128] or None."""
    y = x / np.sqrt((x * x).mean(axis=-1, keepdims=True) + eps)
    return y if weight is None else y * (weight + offset)


def _order(words):
    """Integers that order as the words' values do."""
    w = words.astype(np.int64)
    sign = 1 << (8 * words.dtype.itemsize - 1)
    return np.where(w & sign, -1 - (w & (sign - 1)), w)


def block_keys(pool, bt_row, tag_row, i, dtype):
    """Executed key words [Hkv][16][128] of logical block i."""
    return (fp8.block_bytes if dtype == "e5m2" else paged.block_words)(pool, bt_row, tag_row, i)[0]


def bounds(pool, block_table, tags, seq_lens, known, old, dtype):
    """`old` [B][Hkv][max_blocks][2][128] with the changed blocks' bounds in place."""
    out = np.array(old, copy=True)
    for s, length in enumerate(seq_lens):
        for i in range(int(known[s]) // 16, -(-int(length) // 16)):
            w = block_keys(pool, block_table[s], tags[s], i, dtype)[:, :int(length) - 16 * i]
            order = _order(w)
            for row, pick in ((0, order.argmin(axis=1)), (1, order.argmax(axis=1))):
                out[s, :, i, row] = np.take_along_axis(w, pick[:, None], axis=1)[:, 0]
    return out


def values(words, dtype):
    return fp8.bytes_to_f64(words) if dtype == "e5m2" else encoding.words_to_f64(words, dtype)


def scores(q, lo, hi):
    """q float64 [G][128], lo and hi [n][128]: float64 [n], each sum rounded once."""
    up, down = np.maximum(q, 0.0), np.minimum(q, 0.0)
    up, down = (np.array([math.fsum(c) for c in x.T]) for x in (up, down))
    with np.errstate(invalid="ignore"):
        terms = np.concatenate([up * hi, down * lo], axis=1)
    return np.array([math.fsum(t) if np.isfinite(t).all() else t.sum() for t in terms])


def select(q, bounds_words, seq_lens, budget, sink, recent, dtype):
    """q float64 [B][Hq][128].  Returns (selected, counts)."""
    b, hkv = bounds_words.shape[:2]
    group = q.shape[1] // hkv
    selected, counts = np.full((b, hkv, budget), -1, dtype=np.int32), np.zeros((b, hkv), dtype=np.int32)
    for s, length in enumerate(seq_lens):
        n = -(-int(length) // 16)
        for h in range(hkv):
            x = values(bounds_words[s, h, :n], dtype)
            rank = scores(q[s, h * group:(h + 1) * group], x[:, 0], x[:, 1])
            undefined = np.isnan(rank)   # (above infinity)
            rank[undefined] = np.inf
            ends = [i for i in range(n) if i < sink or i >= n - recent]
            middle = sorted(range(min(sink, n), max(min(sink, n), n - recent)), key=lambda i: (not undefined[i], -rank[i], i))
            chosen = sorted((ends + middle)[:budget])
            selected[s, h, :len(chosen)] = chosen
            counts[s, h] = len(chosen)
    return selected, counts


def listed_tokens(pool, bt_row, tag_row, length, blocks, head, dtype):
    """K and V float64 [tokens][128] of one KV head over the listed blocks that the sequence has."""
    n = -(-int(length) // 16)
    k, v = [], []
    for i in blocks:
        if 0 <= i < n:
            w = (fp8.block_bytes if dtype == "e5m2" else paged.block_words)(pool, bt_row, tag_row, int(i))
            live = min(16, int(length) - 16 * int(i))
            k.append(values(w[0, head, :live], dtype))
            v.append(values(w[1, head, :live], dtype))
    empty = np.zeros((0, 128))
    return np.concatenate(k or [empty]), np.concatenate(v or [empty])


def decode(q, pool, block_table, tags, seq_lens, selected, counts, dtype, scale=None):
    """q float64 [B][Hq][128]; returns float64 of the same shape."""
    b, hq, d = q.shape
    hkv = pool.shape[2]
    scale = 1.0 / math.sqrt(d) if scale is None else scale
    out = np.zeros(q.shape)
    for s in range(b):
        for h in range(hkv):
            k, v = listed_tokens(pool, block_table[s], tags[s], seq_lens[s], selected[s, h, :counts[s, h]], h, dtype)
            if not len(k):
                continue
            for g in range(h * (hq // hkv), (h + 1) * (hq // hkv)):
                x = scale * (k @ q[s, g])
                w = np.exp(x - x.max())
                out[s, g] = w @ v / w.sum()
    return out
