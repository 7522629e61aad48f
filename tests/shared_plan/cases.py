"""Batches that reach the paths of shared-prefix decode which short ones do not, and
what their division has to be for that (an expression of what plan.cpp prints)."""

import numpy as np


def _own(n, most, seed, **at):
    lens = np.random.default_rng(seed).integers(0, most + 1, size=n)
    for s, length in at.items():
        lens[int(s[1:])] = length
    return lens.tolist()


# name: (query heads, KV heads, prefix lengths, group boundaries, own lengths, sequences to compare, what the division is)
CASES = {
    # few workers for each segment: a team's run goes on in the next KV head, its rings used again
    "teams-cross-heads": (64, 4, [6200], [0, 256], _own(256, 40, 1), [0, 9, 130, 255],
                          "not team_aligned and 194 % team_run != 0"),
    "teams-cross-heads-of-two-prefixes": (64, 4, [5200, 4100], [1, 140, 262], _own(263, 40, 2), [0, 1, 100, 139, 140, 261, 262],
                                          "not team_aligned"),
    # more tiles than workers: they come round again
    "tiles-in-rounds": (16, 1, [33 + p % 7 for p in range(600)], list(range(0, 4801, 8)), _own(4800, 20, 3),
                        [0, 7, 8, 2111, 4095, 4096, 4793, 4799], "team_work > team_workers"),
    "tiles-in-rounds-of-two-heads": (32, 2, [64 + p % 40 for p in range(330)], list(range(3, 3 + 8 * 330 + 1, 8)), _own(2650, 10, 4),
                                     [0, 3, 10, 1500, 2642, 2649], "team_work > team_workers"),
    # a stream of more than 64 units of one segment: a prefix's left-over columns, and a long row of own tokens
    "streams-past-a-table": (32, 2, [32768], [0, 330], _own(330, 30, 5, s7=4100), [0, 7, 327, 328, 329], "few_run > 64 and own_run > 64"),
    # all kinds at once, groups of any size, sequences before and behind all of them
    "ragged": (16, 4, [700, 64, 33, 1500, 0, 2570, 31], [2, 5, 5, 6, 18, 18, 58, 59], _own(62, 150, 7, s0=0, s4=0, s8=0), [0, 2, 5, 30, 57, 61],
               "team_workers > 0 and few_workers > 0 and own_workers > 0"),
    # many pieces a column: the merge's waves divide them
    "merge-in-8-ways": (8, 2, [20000], [0, 4], _own(4, 60, 6), [0, 3], "merge_ways == 8"),
}
