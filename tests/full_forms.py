"""Calls that reach every form of full attention's kernels: causal, grouped heads, queries and keys of different lengths, for
every pair of widths.  What each one reaches is asserted on the CPU (test_full_plan.py) and its results on the GPU
(test_gpu_full_forms.py)."""
import random

WIDTHS = (16, 32, 64, 128)
PAIRS = [(d, dv) for d in WIDTHS for dv in WIDTHS]


def _lengths(seed, n, q, k):
    rng = random.Random(seed)
    return [(rng.randint(*q), rng.randint(*k)) for _ in range(n)]


# name: (query heads, key heads, (queries, keys) of each sequence, {plan: (rows of a tile, groups of waves on it, cut into runs)})
FORMS = {
    # many tiles, more than are resident at once, of short streams: one group of waves on a tile
    "many": (16, 8, _lengths(1, 32, (200, 400), (210, 420)) + [(0, 50), (40, 0), (1, 300)],
             {"fwd": (128, 1, False), "dq": (128, 1, False), "dkv": (128, 1, False)}),
    # at most 512 tiles of short streams: one group, the second half of the tiles in the opposite order
    "folded": (8, 4, _lengths(2, 16, (450, 510), (520, 640)),
               {"fwd": (128, 1, False), "dq": (128, 1, False), "dkv": (128, 1, False)}),
    # long streams: two groups; few enough tiles of keys that their streams are cut
    "long": (8, 4, [(4200, 4300), (100, 90)], {"fwd": (128, 2, False), "dq": (128, 2, False), "dkv": (128, 2, True)}),
    # few rows
    "few": (4, 2, [(1, 70), (40, 33), (3, 200), (0, 9)], {"fwd": (32, 1, False), "dq": (32, 1, False), "dkv": (32, 1, False)}),
    # few rows, long streams of either side: cut into runs
    "runs": (4, 2, [(2, 3001), (1, 70), (601, 40), (5, 0)], {"fwd": (32, 1, True), "dq": (32, 1, True), "dkv": (32, 1, True)}),
}


def expected(name, plan, d, dv):
    """The form that a plan has at these widths (at d = d_V = 128 there is no dK/dV kernel with one group of 128 keys)."""
    rows, halves, runs = FORMS[name][3][plan]
    return (rows, 2 if plan == "dkv" and rows == 128 and d + dv == 256 else halves, runs)


def offsets(lengths):
    o = [0]
    for n in lengths:
        o.append(o[-1] + n)
    return o


def case(name):
    """(query heads, key heads, graph_offsets, key_offsets)."""
    H, Hk, lens, _ = FORMS[name]
    return H, Hk, offsets(q for q, _ in lens), offsets(k for _, k in lens)
