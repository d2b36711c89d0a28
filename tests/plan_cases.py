"""Calls over shared rows and chosen blocks, and how the library cuts them: rows of a tile, whether a tile walks through the
shared rows and its sequence's own, whether the keys are cut in parts, and whether rows are read past the caches.
Together they run every tile shape that the plans choose, with whole tiles of several waves, parts and one part."""


def _of(n, batch):
    """Uneven counts, n the first and most."""
    return [max(1, n - (n * ((5 * b) % 4)) // 6) for b in range(batch)]


# name: (dtype, D, KV heads, G, tokens of every sequence, members of every prefix, shared rows, own rows), and
# (rows of a tile, through, parts, once)
SHARED = {
    "bf16_d64_64": (("bf16", 64, 4, 8, [3] * 32, [32], 3000, 100), (64, 0, True, 0)),
    "bf16_d64_64_through": (("bf16", 64, 8, 8, _of(14, 20), [1, 8, 11], 87, 4), (64, 1, False, 0)),
    "bf16_d64_64_through_parts": (("bf16", 64, 4, 4, _of(31, 7), [6], 2065, 9), (64, 1, True, 0)),
    "bf16_d64_128": (("bf16", 64, 8, 2, _of(40, 18), [7, 10, 1], 2955, 37), (128, 0, True, 0)),
    "bf16_d64_128_through": (("bf16", 64, 8, 8, _of(17, 18), [11, 7], 22, 9), (128, 1, False, 0)),
    "bf16_d64_128_through_parts": (("bf16", 64, 8, 4, _of(57, 5), [5], 3773, 0), (128, 1, True, 0)),
    "bf16_d128_128": (("bf16", 128, 8, 1, _of(57, 15), [15], 3054, 0), (128, 0, True, 0)),
    "bf16_d128_128_prompts": (("bf16", 128, 4, 8, [250] * 4, [2, 1], 600, 30), (128, 1, False, 0)),
    "bf16_d128_128_through_parts": (("bf16", 128, 8, 2, _of(77, 8), [8], 1880, 32), (128, 1, True, 0)),
    "f32_d64_128": (("f32", 64, 4, 4, _of(212, 13), [7, 6], 197, 1), (128, 0, True, 0)),
    "f32_d64_128_through": (("f32", 64, 2, 8, _of(19, 5), [5], 32, 0), (128, 1, False, 0)),
    "f32_d64_128_through_parts": (("f32", 64, 8, 4, _of(227, 5), [4], 163, 68), (128, 1, True, 0)),
    "f32_d128_128": (("f32", 128, 1, 8, _of(3, 10), [2, 1, 7], 27, 1), (128, 0, True, 0)),
    "f32_d128_128_through": (("f32", 128, 4, 8, _of(24, 17), [16], 21, 11), (128, 1, False, 0)),
    "f32_d128_128_through_parts": (("f32", 128, 4, 8, _of(36, 6), [6], 387, 15), (128, 1, True, 0)),
}
SHARED_ONCE = {
    "bf16_d128_128": (("bf16", 128, 8, 4, [1] * 50, [16, 10, 14, 7], 16384, 1024), (128, 0, True, 1)),
    "f32_d128_32": (("f32", 128, 8, 4, [1] * 4, [3, 1], 17444, 39), (32, 0, True, 1)),
}

# name: (dtype, D, KV heads, G, tokens, rows, rows of a block, blocks of a list, share)
BLOCKS = {
    "bf16_d64_64": (("bf16", 64, 2, 8, _of(58, 17), 322, 16, 2, 50), (64, 0, False, 0)),
    "bf16_d64_64_parts": (("bf16", 64, 2, 1, _of(62, 19), 1025, 64, 11, 50), (64, 0, True, 0)),
    "bf16_d64_128": (("bf16", 64, 1, 8, _of(15, 21), 3030, 16, 2, 32), (128, 0, False, 0)),
    "bf16_d64_128_parts": (("bf16", 64, 1, 1, _of(127, 24), 2502, 128, 57, 100), (128, 0, True, 0)),
    "bf16_d128_128": (("bf16", 128, 4, 2, _of(52, 19), 137, 16, 52, 50), (128, 0, False, 0)),
    "bf16_d128_128_parts": (("bf16", 128, 1, 4, _of(61, 15), 1557, 128, 48, 50), (128, 0, True, 0)),
    "bf16_d128_128_prompt": (("bf16", 128, 8, 8, [512], 6000, 64, 40, 32), (128, 0, True, 0)),
    "f32_d64_128": (("f32", 64, 8, 4, _of(43, 11), 104, 32, 2, 50), (128, 0, False, 0)),
    "f32_d64_128_parts": (("f32", 64, 2, 8, _of(44, 19), 155, 32, 28, 32), (128, 0, True, 0)),
    "f32_d128_128": (("f32", 128, 4, 8, _of(154, 3), 260, 32, 2, 50), (128, 0, False, 0)),
    "f32_d128_128_parts": (("f32", 128, 2, 2, _of(137, 11), 102, 16, 6, 50), (128, 0, True, 0)),
}
BLOCKS_ONCE = {
    "bf16_d128_32": (("bf16", 128, 8, 1, _of(5, 19), 3572, 64, 85, 50), (32, 0, True, 1)),
    "bf16_d128_128": (("bf16", 128, 8, 1, _of(35, 28), 3457, 128, 18, 50), (128, 0, True, 1)),
    "f32_d128_32": (("f32", 128, 8, 1, _of(9, 10), 3359, 128, 57, 50), (32, 0, True, 1)),
    "f32_d64_32": (("f32", 64, 8, 4, _of(8, 25), 4290, 64, 53, 50), (32, 0, True, 1)),
}
