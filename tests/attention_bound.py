"""What the arithmetic of shared-prefix decode may be off by, element by element.

With t_i = c s_i (c = |scale| log2(e)), w_i = 2^(t_i - max t), L = sum w_i and
out = sum w_i v_i / L, a step u = 2^-24 (half a unit in the last place of 32 bits)
and 2 u for each addition inside the matrix cores, whose rounding is not stated:

* a score is a sum of 128 exact products:        |ds_i| <= 128 * 2u * sum_d |q_d k_id|
* c is three roundings, s c - ref one more, and one where the tail scales first:
                                                 |dt_i| <= c |ds_i| + 5u |t_i| + u max |t|
* a power of two, one unit:                      e_i = ln 2 |dt_i| + 2u   (relative, of w_i)
* a weight enters the product as two halves:     bf16: the head cut off below 2^-7, the
  remainder rounded to 8 bits, 2^-16 of w_i;     fp16: 11 bits each, 2^-23 of w_i, and half of
  the smallest fp16, 2^-25, where w_i is small (the reference never exceeds the maximum, and
  pieces with a lower one are weighed down)
* outputs are 2 n additions of n keys, each      2u of the sum of w_i |v_i| so far at most;
  the sum is n additions of u
* moving the reference and joining pieces: at most one factor and one addition a unit of 32
  keys and a piece, of which a column has at most its units; a factor is a power of two with
  2u of its own:                                 8u a unit, for outputs and sum alike
* the quotient: 2u

The bound is twice the first-order sum of these (for the products of two errors).
"""

import math

import numpy as np

from oracle import encoding, serve

U = 2.0 ** -24


def expected_and_bound(q_words, pool, rows, dtype, scale, group):
    """q_words [Hq][d]; rows: (table row, tag row, tokens) of the prefix and of the
    sequence's own part.  Returns (out, bound), float64 [Hq][d]."""
    half = "fp16" if dtype == "e5m2" else dtype
    q = encoding.words_to_f64(np.asarray(q_words, dtype=np.uint16), half)
    parts = [serve._gather(pool, bt, tg, int(n), dtype) for bt, tg, n in rows if n > 0]
    if not parts:
        return np.zeros(q.shape), np.zeros(q.shape)
    k, v = (np.concatenate([p[i] for p in parts]) for i in (0, 1))
    n = len(k)
    units = sum(-(-int(r[2]) // 32) for r in rows)
    c = abs(scale) * math.log2(math.e)
    split, least = (2.0 ** -16, 0.0) if half == "bf16" else (2.0 ** -23, 2.0 ** -25)
    out, bound = np.empty(q.shape), np.empty(q.shape)
    for h in range(len(q)):
        kh, vh = k[:, h // group], v[:, h // group]
        s, size = kh @ q[h], np.abs(kh) @ np.abs(q[h])
        t = math.copysign(c, scale) * s
        w = np.exp2(t - t.max())
        total = w.sum()
        e = math.log(2) * (c * 128 * 2 * U * size + 5 * U * np.abs(t) + U * np.abs(t).max()) + 2 * U
        out[h] = w @ vh / total
        top = (w * (split + e + 4 * U * n + 8 * U * units) + least) @ np.abs(vh) / total
        below = (w * (e + U * n + 8 * U * units)).sum() / total + 2 * U
        bound[h] = 2 * (top + below * np.abs(out[h]))
    return out, bound
