"""Batches that lead the prompt and shared-prefix attention into each of its work splits, and
the sets that the host plan has to form for them (tests/test_serving_plans.py looks, so that a
change of the plan's rules cannot empty a case)."""

import numpy as np

from paper_2506_01986_amd import synth


def draw(seed, lo, hi, n):
    return [int(v) for v in np.random.default_rng(seed).integers(lo, hi, n)]


def trees_of(kind, B, seed):
    rng = np.random.default_rng(seed)
    one = {"t64": synth.t64, "t16": synth.t16, "single": lambda: synth.chain_tree(1)}
    if kind in one:
        return [one[kind]()] * B
    if kind == "26_or_5":
        return [synth.random_tree(rng, 5 if b % 4 == 3 else 26) for b in range(B)]
    return [synth.random_tree(rng, int(n)) for n in rng.integers(1, 129, B)]


# query heads, KV heads, new tokens, committed rows, prefix rows, groups of one prefix
PROMPTS = {
    # one long context among short prompts: row blocks of 128 cut into chunks, heads 3 and 5 to a KV head
    "split128_g3": (24, 8, [600] + [100] * 40, [5000] + [0] * 40, [0] * 41, None),
    "split128_g5": (40, 8, [333] + draw(7, 1, 120, 40), [6000] + draw(8, 0, 50, 40), [0] * 41, None),
    "split128_prefix": (16, 8, [257] + draw(7, 100, 260, 60), [5000] + draw(8, 0, 50, 60), [700] * 61, [0] + [1] * 60),
    # many short chunks over one prefix: its packed rows in cut blocks of 128
    "packed128": (16, 8, draw(9, 1, 12, 60), draw(10, 0, 300, 60), [3000] * 60, [0] * 60),
    "packed128_table": (16, 8, draw(9, 1, 12, 90), draw(10, 0, 300, 90), [3000] * 90, [i // 45 for i in range(90)]),
    # own rows past 64 beside whole packed blocks, one sequence over a long context
    "packed128_own128": (40, 8, [26] * 30, [4000] + draw(11, 0, 300, 29), [2900] * 30, [0] * 30),
}
# trees, query heads, KV heads, committed rows, prefix rows, groups of one prefix
TREES = {
    "t64_128": ("t64", 64, 8, draw(1, 64, 1024, 10), [2048] * 10, [0] * 10),
    "random_g5_128": ("random", 40, 8, [3000] + draw(2, 0, 300, 17), [300] * 18, [0] * 18),
    "t16_packed128": ("t16", 32, 32, draw(3, 64, 512, 24), [4096] * 24, [0] * 24),
    "t16_packed64": ("t16", 8, 8, draw(3, 0, 200, 24), [1500] * 24, [0] * 24),
    "single_two_prefixes": ("single", 64, 8, draw(4, 16, 512, 64), [8192 - 37 * (i // 32) for i in range(64)], [i // 32 for i in range(64)]),
    "single_table": ("single", 64, 8, draw(3, 0, 200, 100), [3000] * 100, [i // 50 for i in range(100)]),
    "packed128_own128_trees": ("26_or_5", 40, 8, [3000] + draw(12, 0, 300, 27), [2900] * 28, [0] * 28),
}
# the sets that a bf16 batch has to bring: own or packed, rows of a block, whole or cut, "+": merged with a packed prefix
WANT = {
    "split128_g3": {"own 128 cut", "own 128 whole"},
    "split128_g5": {"own 128 cut", "own 128 whole", "own 64 whole"},
    "split128_prefix": {"own 128 cut", "own 128 whole"},
    "packed128": {"packed 128 cut", "own+ 64 whole"},
    "packed128_table": {"packed 128 cut", "own+ 64 whole", "table"},
    "packed128_own128": {"packed 128 whole", "own+ 128 cut", "own+ 128 whole"},
    "t64_128": {"own 128 cut", "own 128 whole"},
    "random_g5_128": {"own 128 cut", "own 128 whole", "own 64 whole"},
    "t16_packed128": {"packed 128 cut", "own+ 64 whole"},
    "t16_packed64": {"packed 64 cut", "own+ 64 whole"},
    "single_two_prefixes": {"packed 128 cut", "own+ 64 whole"},
    "single_table": {"packed 128 cut", "own+ 64 whole", "table"},
    "packed128_own128_trees": {"packed 128 cut", "own+ 128 cut", "own+ 128 whole", "own+ 64 whole"},
}


def nodes(name):
    """Query nodes of a case's sequences."""
    if name in PROMPTS:
        return PROMPTS[name][2]
    return [t.n for t in trees_of(TREES[name][0], len(TREES[name][3]), len(name))]
