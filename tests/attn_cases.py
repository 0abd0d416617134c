"""Lengths that the attention tests share."""

# (heads, KV heads, keys in front, new tokens) of batches with more than 64 items split between CTAs: with two
# tiles of rows to an item, and with one
MANY_SPLIT = [
    (16, 8, [1000 + 251 * b for b in range(12)], [65 + (31 * b) % 136 for b in range(12)]),
    (8, 8, [3000 + 97 * b for b in range(30)], [65 + (13 * b) % 60 for b in range(30)]),
]
