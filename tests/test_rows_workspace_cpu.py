"""A workspace for the largest batch serves every smaller one: its size never decreases.  No GPU: the sizes alone."""
import random

import pytest

from paper_2112_04291_b200 import binding, build


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.lib()


def _need(count, cols):
    """What calls of exactly so many rows and columns take behind the fixed part: tiles of 16, 32, ... positions, two rows of sums and 16 bytes each; or
    (more than 65536 ids) keys and places twice, and 1024 counts for each of the tiles of 1024 to 8192 ids, and in all."""
    lanes = 1
    while lanes < 32 and 8 * lanes < cols:
        lanes *= 2
    chunks, tile = -(-cols // (8 * lanes)), 16
    while -(-count // tile) * chunks * lanes > 32 * 4096 and tile < count:
        tile *= 2
    tiles = -(-count // tile)
    parts = -(-8 * tiles * (cols + 3 & ~3) // 256) * 256 + 16 * tiles
    rounds = min(8, -(-count // 131_072))
    order = 0 if count <= 65_536 else 4 * (-(-4 * count // 256) * 256) + 4096 * -(-count // (1024 * rounds)) + 4096
    return max(parts, order)


COUNTS = sorted({c + d for c in [0, 1, 16, 32, 65_536] + [131_072 * r for r in range(1, 9)] + [2 ** e for e in range(10, 31)] for d in (-17, -1, 0, 1, 17) if 0 <= c + d < 2 ** 31})
COLS = sorted({c + d for c in [8, 16, 32, 64, 128, 256, 512, 1024, 2048, 4096, 65_536, 1 << 20, 1 << 21] for d in (-1, 0, 1)} | {1, 300, 20_000, (1 << 31) - 1})


def test_sizes_do_not_decrease_with_the_ids_or_the_columns(lib):
    fixed = lib.fastsgd_rows_workspace_bytes(0, 1)
    size = {(n, c): lib.fastsgd_rows_workspace_bytes(n, c) for n in COUNTS for c in COLS}
    for n in COUNTS:
        assert all(size[n, a] <= size[n, b] for a, b in zip(COLS, COLS[1:]))
    for c in COLS:
        assert all(size[a, c] <= size[b, c] for a, b in zip(COUNTS, COUNTS[1:]))
    for (n, c), s in size.items():
        assert s >= fixed + _need(n, c)


def test_a_workspace_for_the_largest_batch_serves_every_smaller_one(lib):
    rng = random.Random(1)
    fixed = lib.fastsgd_rows_workspace_bytes(0, 1)
    for _ in range(3_000):
        count, cols = int(2 ** rng.uniform(0, 24)), int(2 ** rng.uniform(0, 15))
        room = lib.fastsgd_rows_workspace_bytes(count, cols)
        products = lib.fastsgd_products_workspace_bytes(count, cols)
        for _ in range(5):
            n, c = rng.randint(1, count), rng.randint(1, cols)
            assert room >= fixed + _need(n, c) and room >= lib.fastsgd_rows_workspace_bytes(n, c)
            assert products >= fixed + 2 * n * c and products >= lib.fastsgd_products_workspace_bytes(n, c)


def test_sizes_stay_near_what_is_needed(lib):
    """No more than 11 MB beyond what the largest call itself takes: 131072 lanes' sums of eight columns each, and 16 bytes a tile."""
    for n in COUNTS:
        for c in COLS:
            if c <= 65_537:
                assert lib.fastsgd_rows_workspace_bytes(n, c) <= lib.fastsgd_rows_workspace_bytes(0, 1) + _need(n, c) + 64 * 131_072 + 16 * 131_072 + 512
