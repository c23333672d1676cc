"""Chunk steps by what their workgroups meet: (query heads, KV heads, tokens held, new tokens) and what
tests/c/chunk_regimes.cpp has to count for them, the least of each: KV heads taken together,
segments of one place that take several, pages of one wave (64 are looked up at once), pages of a
wide segment (512 at once), whole wide row tiles of a workgroup, key tiles of a wide segment."""


def _short(n, seed, most=24, rows=1):
    held = [(seed * 7919 + 13 * i * i + i) % most for i in range(n)]
    return held, [1 + (i * i + seed) % rows for i in range(n)]


STEPS = {
    # short places, one KV head to a wave
    "heads_8": (8, 8, *_short(420, 1), dict(heads=8)),
    "heads_8_of_drafted": (32, 8, *_short(400, 2, rows=8), dict(heads=7)),
    "heads_9": (18, 9, *_short(400, 3, rows=4), dict(heads=8)),
    "heads_16": (16, 16, *_short(420, 4), dict(heads=8, rounds=2)),
    "heads_20_of_7": (140, 20, *_short(300, 5, rows=4), dict(heads=8, rounds=2)),
    "heads_beside_longer": (16, 8, *[x + y for x, y in zip(_short(300, 6, most=140, rows=3), (
        [700, 1023, 1020, 5000, -1, 0, 960, 64], [2, 1, 5, 3, 1, 16, 8, 40]))], dict(heads=4)),
    # few rows over long contexts: a wave looks pages up more than once
    "few_pages_32": (32, 8, [200000, 199999, 150001, 200064, 190000, 200000, 180000, 170000], [4, 1, 8, 3, 8, 2, 5, 7],
                     dict(few=65)),
    "few_pages_64": (32, 8, [200000, 199999, 150001, 200064], [16, 9, 12, 15], dict(few=65)),
    # wide: long runs of pages, several whole row tiles to a workgroup
    "wide_pages": (64, 4, [230000], [256], dict(wide=513, keys=513)),
    "wide_tiles": (64, 4, [0], [4099], dict(whole=2, keys=40)),
    "wide_tiles_of_places": (32, 8, [300, 0, 64, 1000], [3000, 2000, 1999, 1500], dict(whole=2, keys=20)),
    "wide_mixed": (28, 4, [20000, 0, 9000], [2000, 2500, 1], dict(keys=100, wide=100)),
}


def max_context(held, lens):
    return max(h + n for h, n in zip(held, lens)) + 3
