"""Batches whose key ranges are cut, or walked in packed blocks, and merged: fp32 queries over 4-bit pools."""

# query heads, KV heads, new tokens, committed rows, prefix rows, groups of one prefix
MERGES = {
    "cut": (8, 2, [5, 20, 40, 1], [3000, 1500, 700, 2500], [0] * 4, None),
    "packed": (8, 2, [2] * 12, [800] * 12, [1500] * 12, [0] * 12),
    "packed_beside_cut": (4, 4, [3] * 9 + [1], [800] * 9 + [4000], [900] * 9 + [0], [0] * 9 + [1]),
}
