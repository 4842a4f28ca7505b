"""Ids in order, an embedding's lookup and gradient, and experts' products on the GPU against their definitions in 64 bits.

Tolerances: rows_ref states how far 32-bit arithmetic may be off; an output in fewer bits adds half a step of its type.  Where all
values are small whole numbers every sum is exact, and so is the comparison."""
import numpy as np
import pytest
import torch

import rows_ref as ref
from paper_2112_04291_b200 import binding

pytestmark = pytest.mark.gpu

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
MARK = -77.0


def _dev(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return t if dtype is None else t.to(TYPES[dtype])


def _held(a, dtype):
    """float64 values that the type holds"""
    return torch.from_numpy(np.ascontiguousarray(a)).to(TYPES[dtype]).double().numpy()


def _strided(rows, cols, dtype, gap=0, shift=0):
    """A [rows, cols] view with `gap` elements between rows, `shift` elements into its storage; everything is MARK."""
    store = torch.full((shift + rows * (cols + gap) + 64,), MARK, dtype=TYPES[dtype], device="cuda")
    return store, store[shift:shift + rows * (cols + gap)].view(rows, cols + gap)[:, :cols]


def _untouched(store, view):
    rest = store.clone()
    rows, cols = view.shape
    at = view.storage_offset()
    rest[at:at + rows * view.stride(0)].view(rows, -1)[:, :cols] = MARK
    return bool((rest == MARK).all())


def _order(ids, span, distinct=False):
    """order, starts(, distinct, number) with -9 where nothing is written"""
    count = ids.numel()
    order, starts = torch.full((count,), -9, dtype=torch.int32, device="cuda"), torch.full((span + 1,), -9, dtype=torch.int32, device="cuda")
    some, number = torch.full((min(count, span),), -9, dtype=torch.int32, device="cuda"), torch.full((1,), -9, dtype=torch.int32, device="cuda")
    binding.ensure_rows_workspace(count)
    assert binding.order_ids(ids, order, starts, distinct=some if distinct else None, number=number if distinct else None) == 0
    return (order, starts, some, number) if distinct else (order, starts)


def _check_order(ids, span):
    want_order, want_starts, want_distinct = ref.order_ids(ids, span)
    order, starts, distinct, number = (t.cpu().numpy() for t in _order(_dev(ids.astype(np.int32)), span, distinct=True))
    assert np.array_equal(starts, want_starts)
    assert np.array_equal(order[:len(want_order)], want_order) and (order[len(want_order):] == -9).all()
    assert number[0] == len(want_distinct) and np.array_equal(distinct[:number[0]], want_distinct) and (distinct[number[0]:] == -9).all()


# ---- ids in order ----------------------------------------------------------------------------------

@pytest.mark.parametrize("count,span", [(0, 1), (0, 300), (1, 1), (1, 1000), (31, 2), (33, 7), (255, 8), (256, 256), (257, 1023), (1000, 1024), (4097, 1025), (8192, 64), (8193, 128_000),
                                        (20_001, 50_257), (65_535, 999), (65_536, 1 << 20), (65_537, 60), (65_537, 128_000), (300_000, 256), (524_289, 1 << 20), (100_000, 1)])
@pytest.mark.parametrize("kind", ["even", "skewed", "dropped"])
def test_ids_in_order(count, span, kind):
    rng = np.random.default_rng(count + span)
    ids = rng.integers(0, span, count)
    if kind == "skewed":
        ids = np.minimum((span ** rng.random(count)).astype(np.int64), span - 1)
    if kind == "dropped":
        ids[rng.random(count) < 0.3] = -1
        ids[rng.random(count) < 0.1] = span
        ids[rng.random(count) < 0.1] = 2 ** 31 - 1
        ids[rng.random(count) < 0.1] = -2 ** 31
    _check_order(ids, span)


@pytest.mark.parametrize("count,span", [(5000, 400), (5000, 100_000), (100_000, 400), (100_000, 100_000)])
def test_ids_that_are_all_alike_sorted_or_left_out(count, span):
    for ids in (np.full(count, span - 1), np.zeros(count), np.full(count, -1), np.sort(np.arange(count) % span), np.arange(count)[::-1] % span):
        _check_order(ids.astype(np.int64), span)


def test_ids_in_order_are_the_same_every_time():
    ids = torch.randint(0, 3000, (200_000,), dtype=torch.int32, device="cuda")
    first = _order(ids, 3000)
    for _ in range(20):
        assert all(torch.equal(a, b) for a, b in zip(first, _order(ids, 3000)))


# ---- an embedding's lookup -----------------------------------------------------------------------------

PAIRS_OF_TYPES = [("fp32", "fp32"), ("fp32", "bf16"), ("fp32", "fp16"), ("bf16", "bf16"), ("bf16", "fp32"), ("fp16", "fp16"), ("fp16", "fp32")]


@pytest.mark.parametrize("dtype,out", PAIRS_OF_TYPES)
@pytest.mark.parametrize("tokens,vocab,cols,gap,shift", [(0, 5, 8, 0, 0), (1, 1, 1, 0, 0), (1, 7, 4096, 0, 0), (65, 40, 8, 0, 0), (33, 100, 12, 4, 0), (50, 9, 257, 0, 1), (7, 300, 1001, 3, 5),
                                                         (300, 50, 264, 8, 8), (5000, 1000, 72, 0, 0), (3, 4, 20_000, 0, 0), (5, 4, 130, 6, 0)])
def test_lookup(dtype, out, tokens, vocab, cols, gap, shift):
    rng = np.random.default_rng(cols)
    table = _held(rng.normal(0, 1, (vocab, cols)), dtype)
    ids = rng.integers(-1, vocab + 1, tokens)
    _, view = _strided(vocab, cols, dtype, gap, shift)
    view.copy_(torch.from_numpy(table))
    store, rows = _strided(tokens, cols, out, gap, shift)
    for scale in (1.0, -0.3):
        assert binding.embedding(view, _dev(ids.astype(np.int32)), rows, scale=scale) == 0
        want = ref.embedding(table, ids, float(np.float32(scale)))
        assert (np.abs(rows.double().cpu().numpy() - want) <= ref.U * np.abs(want) * (scale != 1.0) + (ref.rounding(want, out) if scale != 1.0 or out != dtype else 0.0)).all()
        assert tokens == 0 or _untouched(store, rows)


def test_lookup_passes_infinities_and_nan_on_and_padding_reads_no_row():
    table = torch.tensor([[float("inf"), float("nan"), -float("inf"), 1.0] * 3] * 2, device="cuda")
    out = torch.empty((3, 12), device="cuda")
    assert binding.embedding(table, torch.tensor([1, -1, 2], dtype=torch.int32, device="cuda"), out, scale=0.5) == 0
    assert torch.equal(out[0].nan_to_num(nan=7.0), (table[0] * 0.5).nan_to_num(nan=7.0)) and (out[1:] == 0).all()


# ---- its gradient ------------------------------------------------------------------------------------

def _ids(rng, tokens, vocab, kind):
    if kind == "alike":
        return np.full(tokens, vocab // 2)
    ids = np.minimum((vocab ** rng.random(tokens)).astype(np.int64), vocab - 1) if kind == "skewed" else rng.integers(0, vocab, tokens)
    if kind == "padded":
        ids[rng.random(tokens) < 0.5] = -1
        ids[rng.random(tokens) < 0.05] = vocab
    return ids


def _check_gradient(rng, tokens, vocab, cols, dtype, out, kind, gap=0, shift=0, scale=0.3):
    grad = _held(rng.normal(0, 1, (tokens, cols)), dtype)
    ids = _ids(rng, tokens, vocab, kind)
    _, view = _strided(tokens, cols, dtype, gap, shift)
    view.copy_(torch.from_numpy(grad))
    dev_ids = _dev(ids.astype(np.int32))
    binding.ensure_rows_workspace(tokens, cols)
    order, starts, distinct, number = _order(dev_ids, vocab, distinct=True)
    binding.ensure_rows_workspace(tokens, cols)
    store, table = _strided(vocab, cols, out, gap, shift)
    assert binding.embedding_backward(view, dev_ids, order, starts, table, scale=scale) == 0
    want, size, terms = ref.embedding_backward(grad, ids, vocab, float(np.float32(scale)))
    off = ref.sum_error(size, terms)
    assert (np.abs(table.double().cpu().numpy() - want) <= off + ref.rounding(np.abs(want) + off, out)).all()
    assert _untouched(store, table)
    if out != "fp32":
        return
    most = min(tokens, vocab)
    keys, values = torch.full((most + 1, cols), -9, dtype=torch.int32, device="cuda"), torch.full((most + 1, cols), MARK, device="cuda")
    assert binding.embedding_backward_pairs(view, dev_ids, order, starts, distinct, number, keys[:most], values[:most], scale=scale) == 0
    n = int(number.item())
    occur = distinct[:n].long()
    assert torch.equal(keys[:n].long(), occur[:, None] * cols + torch.arange(cols, device="cuda"))
    assert torch.equal(values[:n], table[occur])                             # the same sums in the same order
    assert (keys[n:] == -9).all() and (values[n:] == MARK).all()


@pytest.mark.parametrize("dtype,out", PAIRS_OF_TYPES)
@pytest.mark.parametrize("tokens,vocab,cols,kind", [(1, 1, 1, "even"), (1, 9, 8, "even"), (15, 4, 16, "even"), (16, 4, 16, "even"), (17, 4, 264, "skewed"), (33, 1, 24, "alike"), (300, 50, 1001, "padded"),
                                                    (1000, 3, 64, "even"), (2000, 700, 520, "skewed"), (4097, 40, 8, "alike"), (3000, 10_000, 40, "padded"), (64, 100, 4096, "padded")])
def test_gradient(dtype, out, tokens, vocab, cols, kind):
    _check_gradient(np.random.default_rng(tokens + cols), tokens, vocab, cols, dtype, out, kind)


@pytest.mark.parametrize("dtype,out", PAIRS_OF_TYPES)
@pytest.mark.parametrize("gap,shift,cols", [(0, 1, 40), (3, 0, 37), (8, 8, 264), (4, 4, 20), (2, 0, 6)])
def test_gradient_of_rows_at_any_place(dtype, out, gap, shift, cols):
    _check_gradient(np.random.default_rng(cols), 200, 30, cols, dtype, out, "skewed", gap, shift)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("tokens,vocab,cols", [(70_000, 5, 300), (70_000, 1000, 256), (40_000, 2, 1024), (9_000, 400, 4100)])
def test_gradient_of_many_tokens(dtype, tokens, vocab, cols):
    _check_gradient(np.random.default_rng(tokens), tokens, vocab, cols, dtype, "fp32", "skewed")


def test_gradient_of_no_tokens_and_of_padding_alone_is_zero():
    for tokens in (0, 50):
        ids = torch.full((tokens,), -1, dtype=torch.int32, device="cuda")
        order, starts = _order(ids, 20)
        binding.ensure_rows_workspace(max(tokens, 1), 40)
        table = torch.full((20, 40), MARK, device="cuda")
        grad = torch.full((tokens, 40), float("nan"), device="cuda")
        assert binding.embedding_backward(grad, ids, order, starts, table) == 0
        assert (table == 0).all()


def test_gradient_passes_nan_to_its_own_row_alone():
    ids = torch.arange(200, dtype=torch.int32, device="cuda") % 40
    ids[7] = -1
    grad = torch.ones((200, 24), device="cuda")
    grad[5, 3], grad[7, :] = float("nan"), float("nan")
    order, starts = _order(ids, 40)
    binding.ensure_rows_workspace(200, 24)
    table = torch.empty((40, 24), device="cuda")
    assert binding.embedding_backward(grad, ids, order, starts, table) == 0
    want = torch.full((40, 24), 5.0, device="cuda")
    want[7] = 4.0
    want[5, 3] = float("nan")
    assert torch.equal(table.nan_to_num(nan=-1.0), want.nan_to_num(nan=-1.0))


def test_gradient_is_the_same_every_time():
    ids = (torch.rand((30_000,), device="cuda") ** 3 * 500).to(torch.int32)
    grad = torch.randn((30_000, 72), device="cuda")
    order, starts = _order(ids, 500)
    binding.ensure_rows_workspace(30_000, 72)
    first, again = torch.empty((500, 72), device="cuda"), torch.empty((500, 72), device="cuda")
    assert binding.embedding_backward(grad, ids, order, starts, first) == 0
    for _ in range(20):
        assert binding.embedding_backward(grad, ids, order, starts, again) == 0
        assert torch.equal(first, again)


# ---- experts' products ---------------------------------------------------------------------------------

def _routed(rng, tokens, experts, k, dropped=0.1, idle=()):
    selected = np.argsort(rng.random((tokens, experts)) + 0.3 * rng.random(experts), axis=1)[:, :k]
    selected[rng.random((tokens, k)) < dropped] = -1
    for e in idle:
        selected[selected == e] = -1
    return selected


def _whole(rng, shape, dtype, whole):
    return rng.integers(-3, 4, shape).astype(np.float64) if whole else _held(rng.normal(0, 1, shape), dtype)


def _weights(a, dtype, gap=0, between=0):
    experts, outs, ins = a.shape
    store = torch.full((experts * (outs * (ins + gap) + between),), MARK, dtype=TYPES[dtype], device="cuda")
    view = store.view(experts, -1)[:, :outs * (ins + gap)].unflatten(1, (outs, ins + gap))[:, :, :ins]
    view.copy_(torch.from_numpy(a))
    return store, view


def _near(got, want, size, terms, out, whole):
    """exact for whole numbers (sums below 2^24), else within the bounds"""
    off = 0.0 if whole else ref.product_error(size, terms)
    return (np.abs(got - want) <= off + (ref.rounding(np.abs(want) + off, out) if out != "fp32" or not whole else 0.0)).all()


def _check_products(rng, tokens, experts, k, ins, outs, dtype, out, whole, gap=0, between=0, sorted_rows=False, idle=(), dropped=0.1):
    selected = _routed(rng, tokens, experts, k, dropped, idle)
    rows = tokens * k
    order, starts = _order(_dev(selected.astype(np.int32)), experts)
    want_order, want_starts, _ = ref.order_ids(selected, experts)
    kept = len(want_order)
    source = np.zeros(rows, dtype=np.int64)
    source[:kept] = want_order // k
    x, w = _whole(rng, (tokens, ins), dtype, whole), _whole(rng, (experts, outs, ins), dtype, whole)
    gy = _whole(rng, (rows, outs), dtype, whole)
    if sorted_rows:                                       # no order: x has been sorted by the caller
        x, source, order, per_row = x[source], np.arange(rows), None, 1
    else:
        per_row = k
    gy_held = gy.copy()
    gy_held[kept:] = np.nan                               # rows that belong to no expert
    x_held = x.copy()
    if sorted_rows:
        x_held[kept:] = np.nan
    _, dx = _strided(x.shape[0], ins, dtype, gap)
    dx.copy_(torch.from_numpy(x_held))
    _, dgy = _strided(rows, outs, dtype, gap)
    dgy.copy_(torch.from_numpy(gy_held))
    _, dw = _weights(w, dtype, gap, between)

    binding.ensure_products_workspace(rows, ins)
    store, y = _strided(rows, outs, out, gap)
    assert binding.expert_product(dx, dw, starts, y, order=order, per_row=per_row) == 0
    want, size = ref.products(x, source, want_starts, w)
    got = y.double().cpu().numpy()
    assert _near(got[:kept], want[:kept], size[:kept], ins, out, whole)
    assert (got[kept:] == MARK).all() and _untouched(store, y)

    store, gx = _strided(rows, ins, out, gap)
    assert binding.expert_product_backward_input(dgy, dw, starts, gx) == 0
    want, size = ref.products_input(gy, want_starts, w)
    got = gx.double().cpu().numpy()
    assert _near(got[:kept], want[:kept], size[:kept], outs, out, whole)
    assert (got[kept:] == MARK).all() and _untouched(store, gx)

    store, gw = _weights(np.full((experts, outs, ins), MARK), out, gap, between)
    assert binding.expert_product_backward_weights(dgy, dx, starts, gw, order=order, per_row=per_row) == 0
    want, size = ref.products_weights(gy, x, source, want_starts)
    terms = np.diff(want_starts)[:, None, None]
    assert _near(gw.double().cpu().numpy(), want, size, terms, out, whole)
    gw.fill_(MARK)
    assert bool((store == MARK).all())


PRODUCTS = [  # tokens, experts, k, ins, outs
    (1, 1, 1, 8, 8), (1, 4, 2, 64, 128), (3, 8, 2, 72, 136), (16, 8, 2, 512, 264), (40, 1, 1, 200, 56), (100, 5, 3, 128, 384), (300, 3, 1, 264, 512), (257, 2, 2, 320, 1000), (700, 60, 4, 120, 88),
    (1030, 4, 2, 648, 640), (50, 300, 3, 64, 72)]


@pytest.mark.parametrize("dtype,out", [("bf16", "bf16"), ("fp16", "fp16"), ("bf16", "fp32"), ("fp16", "fp32")])
@pytest.mark.parametrize("tokens,experts,k,ins,outs", PRODUCTS)
@pytest.mark.parametrize("whole", [True, False])
def test_products(dtype, out, tokens, experts, k, ins, outs, whole):
    _check_products(np.random.default_rng(tokens + ins), tokens, experts, k, ins, outs, dtype, out, whole)


@pytest.mark.parametrize("dtype,out", [("bf16", "bf16"), ("fp16", "fp16"), ("bf16", "fp32")])
@pytest.mark.parametrize("tokens,experts,k,ins,outs", [(1, 1, 1, 4096, 264), (8, 1, 1, 8200, 520), (3, 4, 2, 2056, 1032), (40, 2, 1, 1032, 3080), (300, 1, 1, 2048, 1288), (5000, 1, 1, 64, 72), (9000, 3, 1, 272, 136),
                                                       (20_000, 2, 2, 8, 264)])
@pytest.mark.parametrize("whole", [True, False])
def test_products_of_few_tiles_and_long_contractions(dtype, out, tokens, experts, k, ins, outs, whole):
    _check_products(np.random.default_rng(tokens + ins), tokens, experts, k, ins, outs, dtype, out, whole)


@pytest.mark.parametrize("tokens,experts,k,ins,outs", [(3, 8, 2, 72, 136), (257, 2, 2, 320, 1000), (700, 60, 4, 120, 88)])
@pytest.mark.parametrize("gap,between", [(8, 0), (0, 8), (24, 16)])
def test_products_of_strided_matrices(tokens, experts, k, ins, outs, gap, between):
    _check_products(np.random.default_rng(gap), tokens, experts, k, ins, outs, "bf16", "bf16", True, gap, between)


@pytest.mark.parametrize("tokens,experts,k,ins,outs", PRODUCTS)
def test_products_of_rows_that_are_sorted_already(tokens, experts, k, ins, outs):
    _check_products(np.random.default_rng(ins), tokens, experts, k, ins, outs, "fp16", "fp32", True, sorted_rows=True)


@pytest.mark.parametrize("dropped,idle", [(0.0, ()), (1.0, ()), (0.0, (0, 1, 5)), (0.5, (7,))])
def test_products_where_experts_have_no_rows(dropped, idle):
    _check_products(np.random.default_rng(5), 200, 8, 2, 136, 264, "bf16", "fp32", True, idle=idle, dropped=dropped)
