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


# ---- outputs on top of whole numbers that the call reads -------------------------------------------

A, B, C, D, E, F = (1 << 20 | i << 24 for i in range(1, 7))      # never dereferenced: the checks fail before any launch


def _matrix(data, rows, cols, kind=binding.BF16):
    return binding.Matrix(data, rows, cols, cols, kind, 0)


def test_an_order_does_not_lie_on_its_ids_or_its_starts(lib):
    def call(ids=A, order=B, starts=C, distinct=D, number=E):
        return lib.fastsgd_order_ids(ids, 70_000, 500, order, starts, distinct, number, None)
    at = dict(ids=A, order=B, starts=C, distinct=D, number=E)
    size = dict(ids=70_000, order=70_000, starts=501, distinct=500, number=1)
    for one in at:
        for other in at:
            if one != other:
                assert call(**{one: at[other] + 4 * (size[other] - 1)}) == binding.E_BAD_PARAM
                assert call(**{one: at[other] - 4 * (size[one] - 1)}) == binding.E_BAD_PARAM
    assert call(order=A, distinct=None, number=None) == binding.E_BAD_PARAM


def test_rows_do_not_lie_on_the_ids_that_choose_them(lib):
    table, grad = _matrix(A, 100, 16), _matrix(B, 10, 16)
    for ids in (B, B + 16 * 2 * 10 - 4):
        assert lib.fastsgd_embedding(table, ids, 1.0, grad, None) == binding.E_BAD_PARAM
    for i in range(3):
        words = [C, D, E]
        words[i] = A + 100 * 32 - 4
        assert lib.fastsgd_embedding_backward(grad, *words, 1.0, table, None) == binding.E_BAD_PARAM
    for on in (A, F):
        for i in range(5):
            words = [C, C + 4096, D, D + 4096, E]
            words[i] = on + 4 * 10 * 16 - 4
            assert lib.fastsgd_embedding_backward_pairs(grad, *words, 100, 1.0, A, F, 10, None) == binding.E_BAD_PARAM


def test_products_do_not_lie_on_the_order_or_the_starts(lib):
    x, y, w = _matrix(A, 10, 16), _matrix(B, 20, 24), binding.Experts(C, 4, 24, 16, 16, 24 * 16, binding.BF16, 0)
    for order, starts in ((B + 4, D), (D, B + 20 * 48 - 4)):
        assert lib.fastsgd_expert_product(x, order, 2, starts, w, y, None) == binding.E_BAD_PARAM
    assert lib.fastsgd_expert_product_backward_input(y, E + 20 * 32 - 4, w, _matrix(E, 20, 16), None) == binding.E_BAD_PARAM
    for order, starts in ((C + 4, D), (D, C + 4 * 24 * 32 - 4)):
        assert lib.fastsgd_expert_product_backward_weights(y, x, order, 2, starts, w, None) == binding.E_BAD_PARAM
