"""Top logits, the distillation loss and the balance loss on the GPU against their definitions in 64 bits.

Tolerances: loss_ref states how far 32-bit arithmetic may be off; an output in fewer bits adds half a step of its type."""
import itertools

import numpy as np
import pytest
import torch

import loss_ref as ref
from paper_2112_04291_b200 import binding

pytestmark = pytest.mark.gpu

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
MARK = -77.0          # what lies between rows and behind the last


def _dev(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return t if dtype is None else t.to(dtype)


def _logits(rng, rows, cols, dtype, scale=2.0):
    """float64 values that the type holds exactly"""
    return torch.from_numpy(rng.normal(0, scale, (rows, cols))).to(TYPES[dtype]).double().numpy()


def _strided(a, dtype, gap=0, shift=0):
    """A [rows, cols] view on the GPU with `gap` elements between rows, `shift` elements into its storage; all else is MARK."""
    rows, cols = a.shape
    store = torch.full((shift + rows * (cols + gap) + 64,), MARK, dtype=TYPES[dtype], device="cuda")
    view = store[shift:shift + rows * (cols + gap)].view(rows, cols + gap)[:, :cols]
    view.copy_(torch.from_numpy(a))
    return store, view


def _untouched(store, view):
    """Whether everything of the storage but the view is MARK."""
    rest = store.clone()
    rows, cols = view.shape
    at = view.storage_offset()
    rest[at:at + rows * view.stride(0)].view(rows, -1)[:, :cols] = MARK if rows else MARK
    return bool((rest == MARK).all())


def _same(a, b):
    return torch.equal(a.view(torch.int32 if a.element_size() == 4 else torch.int16), b.view(torch.int32 if b.element_size() == 4 else torch.int16))


# ---- top logits ------------------------------------------------------------------------------------

def _run_top(view, k, temperature):
    rows = view.shape[0]
    keys = torch.full((rows, k), -9, dtype=torch.int32, device="cuda")
    values = torch.full((rows, k), MARK, dtype=view.dtype, device="cuda")
    lse, tail = torch.full((rows,), MARK, device="cuda"), torch.full((rows,), MARK, device="cuda")
    assert binding.top_logits(view, keys, values, temperature=temperature, lse=lse, tail=tail) == 0
    return keys, values, lse, tail


def _check_top(z, view, k, temperature=1.0):
    keys, values, lse, tail = _run_top(view, k, temperature)
    want_keys, want_values, want_lse, want_tail = ref.top(z, k, temperature)
    assert np.array_equal(keys.cpu().numpy(), want_keys)
    got = values.double().cpu().numpy()
    assert np.array_equal(got, want_values, equal_nan=True)
    got_lse, got_tail = lse.double().cpu().numpy(), tail.double().cpu().numpy()
    fine = np.isfinite(want_lse)
    assert np.array_equal(got_lse[~fine], want_lse[~fine], equal_nan=True) and np.array_equal(got_tail[~fine], want_tail[~fine], equal_nan=True)
    # as loss_ref.distill: an exponential EX2 + 3 U |d|, a sum (cols / 512 + 24) U; m / T, a logarithm and their sum, each a half step
    for r in np.flatnonzero(fine):
        x = z[r][np.isfinite(z[r])]
        d = min((x.max() - x.min()) / temperature, 104.0)
        unit = ref.EX2 + (3.0 * d + z.shape[1] / 512.0 + 40.0) * ref.U
        assert abs(got_lse[r] - want_lse[r]) <= unit + 4.0 * ref.U * (abs(x.max()) / temperature + np.log(z.shape[1]) + abs(want_lse[r])), r
        assert abs(got_tail[r] - want_tail[r]) <= 2.0 * unit * want_tail[r] + 2.0 ** -126, r


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("rows,cols,k,temperature", [
    (1, 1, 1, 1.0), (2, 3, 2, 1.0), (3, 33, 33, 0.5), (5, 1000, 64, 2.0), (70, 256, 8, 1.0), (33, 60, 6, 1.0), (2, 1024, 1024, 1.0), (2, 1023, 32, 1.0),
    (2, 1025, 33, 1.0), (1, 4097, 1000, 3.0), (2, 50_257, 300, 1.0), (1, 128_000, 20, 1.0), (3, 70_001, 1024, 1.0), (300, 2_049, 5, 1.0), (1, 300_001, 64, 0.7)])
def test_top_logits(dtype, rows, cols, k, temperature):
    rng = np.random.default_rng(cols + k)
    z = _logits(rng, rows, cols, dtype)
    _check_top(z, _dev(z, TYPES[dtype]), k, temperature)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("gap,shift", [(0, 1), (3, 0), (5, 7), (8, 8)])
@pytest.mark.parametrize("cols,k", [(40, 5), (517, 40), (9_001, 100)])
def test_top_logits_of_rows_at_any_place(dtype, gap, shift, cols, k):
    z = _logits(np.random.default_rng(shift + cols), 5, cols, dtype)
    store, view = _strided(z, dtype, gap, shift)
    _check_top(z, view, k)
    assert _untouched(store, view)


def _hard_rows(cols):
    rng = np.random.default_rng(cols)
    base = rng.normal(0, 2, cols)
    few = np.full(cols, -np.inf)
    few[rng.choice(cols, min(cols, 5), replace=False)] = rng.normal(0, 1, min(cols, 5))
    nan = base.copy()
    nan[rng.choice(cols, min(cols, 40), replace=False)] = np.nan
    inf = base.copy()
    inf[cols // 2], inf[cols // 3] = np.inf, -np.inf
    signs = np.where(rng.random(cols) < 0.5, 0.0, -0.0)
    comb = base.copy()
    comb[::64] += 30.0                                                        # the largest all in a few threads' share
    ridge = base.copy()
    ridge[cols // 2:cols // 2 + 700] = 50.0                                   # ... and many equal ones next to each other
    return np.stack([np.zeros(cols), np.sort(base), np.sort(base)[::-1], np.round(base), few, np.full(cols, -np.inf), nan, inf, signs, comb, ridge,
                     np.full(cols, -60_000.0), np.where(np.arange(cols) % 2, 1.0, -np.inf)])


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("cols,k", [(8, 8), (256, 8), (1000, 32), (1000, 500), (20_011, 64), (20_011, 1024), (130_001, 64)])
def test_top_logits_of_ties_infinities_nan_and_sorted_rows(dtype, cols, k):
    z = torch.from_numpy(_hard_rows(cols).copy()).to(TYPES[dtype]).double().numpy()
    _check_top(z, _dev(z, TYPES[dtype]), k)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("cols,k", [(50_001, 64), (50_001, 700), (200_003, 300)])
def test_top_logits_sums_are_the_same_every_time(dtype, cols, k):
    """Rows of the same values at places of the same alignment: the order in which a block finds its pairs must not show."""
    row = _dev(_logits(np.random.default_rng(cols), 1, cols, dtype), TYPES[dtype])
    row[0, 100:140] = row[0, 200:240]                                         # (ties)
    z = torch.empty((200, cols + (-cols) % 8), dtype=TYPES[dtype], device="cuda")[:, :cols]
    z.copy_(row.expand(200, cols))
    first = _run_top(z, k, 1.0)
    for got in (first, _run_top(z, k, 1.0)):
        for a, b in zip(got, first):
            assert _same(a, b[:1].expand_as(b).contiguous())


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("rows,cols,k,gap,shift", [(8_192, 1, 1, 0, 0), (8_300, 7, 3, 2, 5), (8_191, 8, 2, 0, 0), (8_192, 8, 8, 0, 8), (16_390, 16, 2, 0, 0), (16_401, 13, 13, 0, 1),
                                                   (32_800, 32, 4, 0, 4), (32_769, 27, 9, 5, 3)])
def test_top_logits_of_many_short_rows(dtype, rows, cols, k, gap, shift):
    z = _logits(np.random.default_rng([rows, cols, k]), rows, cols, dtype)
    z[::7, cols // 2:] = z[::7, :1]                        # equal values
    z[3::11, :cols // 2] = -np.inf
    z[5], z[rows - 1, 0], z[rows - 2, cols - 1] = -np.inf, np.nan, np.inf
    store, view = _strided(z, dtype, gap, shift)
    _check_top(z, view, k, 0.8)
    assert _untouched(store, view)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("cols,k", [(65, 6), (100, 16), (128, 16), (129, 4), (256, 16), (257, 5), (777, 16), (1024, 9)])
def test_top_logits_of_few_columns_with_few_different_values(dtype, cols, k):
    """From all different to all alike: few and many values as large as the k-th."""
    rng = np.random.default_rng([cols, k])
    z = _logits(rng, 60, cols, dtype)
    for r in range(60):
        levels = _logits(rng, 1, 1 + r // 2, dtype)[0]
        if r % 2 == 0:
            z[r] = levels[rng.integers(0, len(levels), cols)]
    z[1, 3:], z[3, 1::2], z[7, 32:] = -np.inf, -np.inf, -np.inf
    _check_top(z, _strided(z, dtype)[1], k)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("cols,k", [(40, 6), (5_000, 6), (70_000, 200)])
def test_top_logits_have_one_zero_and_one_nan(dtype, cols, k):
    z = torch.full((2, cols), -1.0, device="cuda").to(TYPES[dtype])
    words = z.view(torch.int32 if dtype == "fp32" else torch.int16)
    words[:, 5] = -2 ** 31 if dtype == "fp32" else -2 ** 15                    # -0
    z[:, 9] = 0.0
    words[1, 7], words[1, 11] = (-3, 0x7FC00123) if dtype == "fp32" else (-3, 0x7FFD)      # NaN, of either sign
    keys, values, lse, tail = _run_top(z, k, 1.0)
    assert keys[0, :2].tolist() == [5, 9] and keys[1, :4].tolist() == [7, 11, 5, 9]
    bits = values.view(words.dtype)
    assert bits[0, :2].tolist() == [0, 0] and bits[1, 2:4].tolist() == [0, 0]
    assert bool(values[1, :2].isnan().all()) and bits[1, 0] == bits[1, 1]
    assert bool((values[:, 4:] == -1.0).all()) and bool(lse[1].isnan()) and bool(tail[1].isnan())


def test_calls_on_two_streams_at_once():
    """They share nothing: neither a workspace nor anything the library keeps."""
    gen = torch.Generator(device="cuda").manual_seed(4)
    z = [torch.randn((700, 50_001), generator=gen, device="cuda").to(torch.bfloat16) for _ in range(2)]
    x = [torch.randn((5_000, 60), generator=gen, device="cuda") for _ in range(2)]

    def all_calls(i):
        keys, values = torch.empty((700, 64), dtype=torch.int32, device="cuda"), torch.empty((700, 64), dtype=torch.bfloat16, device="cuda")
        lse, tail, loss, grad = torch.empty(700, device="cuda"), torch.empty(700, device="cuda"), torch.empty(700, device="cuda"), torch.empty_like(z[i])
        chosen, weights = torch.empty((5_000, 6), dtype=torch.int32, device="cuda"), torch.empty((5_000, 6), device="cuda")
        counts, counted, slope = torch.empty((1, 60), dtype=torch.int32, device="cuda"), torch.empty(1, dtype=torch.int32, device="cuda"), torch.empty_like(x[i])
        assert binding.top_logits(z[i], keys, values, lse=lse, tail=tail) == 0
        assert binding.distill_loss(z[1 - i], keys, values, loss=loss, grad=grad, tail=tail) == 0
        assert binding.top_logits(x[i], chosen, weights) == 0
        assert binding.expert_counts(chosen, counts, counted) == 0
        assert binding.balance_loss(x[i], counts, counted, grad=slope) == 0
        return keys, values, lse, tail, loss, grad, chosen, weights, counts, counted, slope

    alone = [all_calls(i) for i in range(2)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(5):
        both = []
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                both.append(all_calls(i))
        torch.cuda.synchronize()
        for i in range(2):
            assert all(_same(a, b) for a, b in zip(alone[i], both[i]))


def test_top_logits_optional_outputs_and_no_rows():
    z = torch.randn(3, 500, device="cuda")
    keys, values = torch.empty(3, 4, dtype=torch.int32, device="cuda"), torch.empty(3, 4, device="cuda")
    assert binding.top_logits(z, keys, values) == 0
    want = z.topk(4, dim=1)
    assert torch.equal(keys.long(), want.indices) and torch.equal(values, want.values)
    only = torch.empty(3, device="cuda")
    assert binding.top_logits(z, keys, values, tail=only) == 0 and torch.equal(only, _run_top(z, 4, 1.0)[3])
    assert binding.top_logits(z, keys, values, lse=only) == 0 and torch.equal(only, _run_top(z, 4, 1.0)[2])
    launches = binding.launch_count()
    assert binding.top_logits(z[:0], keys[:0], values[:0]) == 0 and binding.launch_count() == launches


# ---- distillation -----------------------------------------------------------------------------------

def _teacher(rng, rows, cols, k, ragged=False):
    keys = np.stack([rng.choice(cols, k, replace=False) for _ in range(rows)]).astype(np.int32)
    values = rng.normal(0, 2, (rows, k)).astype(np.float32)
    if ragged:
        for r in range(rows):
            keys[r, rng.integers(1, k + 1):] = (-1, cols, 1 << 30, -(1 << 31))[r % 4]
    return keys, values


def _run_distill(view, keys, values, temperature, tail, weight, grad_type, in_place=False, want_loss=True):
    rows, cols = view.shape
    loss = torch.full((rows,), MARK, device="cuda") if want_loss else None
    stats = torch.full((rows, 2), MARK, device="cuda")
    grad = None
    if grad_type is not None:
        grad = view if in_place else torch.full((rows, cols), MARK, dtype=TYPES[grad_type], device="cuda")
    assert binding.distill_loss(view, keys, values, loss=loss, grad=grad, temperature=temperature, tail=tail, weight=weight, stats=stats) == 0
    return loss, grad, stats


def _check_distill(z, dtype, keys, values, temperature=1.0, tail=None, weight=None, values_type="fp32", view=None, grad_types=None):
    """Loss and gradient of every form of the call: forward alone, with the gradient (in each type, in place), backward from the stats."""
    rows = z.shape[0]
    vals = torch.from_numpy(np.asarray(values)).to(TYPES[values_type])
    want_loss, want_grad, grad_err, loss_err = ref.distill(z, keys, vals.double().numpy(), temperature, tail, weight)
    view = _dev(z, TYPES[dtype]) if view is None else view
    k_, v_ = _dev(keys.astype(np.int32)), vals.cuda()
    t_ = None if tail is None else _dev(tail.astype(np.float32))
    w_ = None if weight is None else _dev(weight.astype(np.float32))

    def check_loss(got):
        got = got.double().cpu().numpy()
        fine = np.isfinite(want_loss)
        assert np.array_equal(got[~fine], want_loss[~fine], equal_nan=True)
        off = np.abs(got - want_loss)[fine]
        assert np.all(off <= loss_err[fine] + 2.0 ** -140), (off - loss_err[fine]).max()

    def check_grad(got, kind, up=None):
        got = got.double().cpu().numpy()
        u = np.ones(rows) if up is None else up
        want, err = want_grad * u[:, None], grad_err * np.abs(u)[:, None]
        # half a step of the type, its smallest step, and what the exponential flushes to zero
        tol = err + ref.HALF_STEP[kind] * (np.abs(want) + err) + ref.LEAST[kind] + 2.0 ** -120
        fine = np.isfinite(want)
        assert np.array_equal(np.isnan(got), np.isnan(want))
        off = np.abs(got - want)[fine]
        assert np.all(off <= tol[fine]), ((off - tol[fine]).max(), off.max())

    loss, _, stats = _run_distill(view, k_, v_, temperature, t_, w_, None)
    check_loss(loss)
    up = np.random.default_rng(rows).normal(0, 1, rows).astype(np.float32)
    for kind in grad_types or dict.fromkeys([dtype, "fp32"]):
        loss2, grad, stats2 = _run_distill(view, k_, v_, temperature, t_, w_, kind)
        check_loss(loss2)                                  # (the sums have another order than without a gradient)
        check_grad(grad, kind)
        back = torch.full_like(grad, MARK)
        assert binding.distill_loss_backward(view, k_, v_, stats, back, temperature=temperature, tail=t_, weight=w_) == 0
        check_grad(back, kind)
        assert binding.distill_loss_backward(view, k_, v_, stats2, back, grad_loss=_dev(up), temperature=temperature, tail=t_, weight=w_) == 0
        check_grad(back, kind, up.astype(np.float64))
        if kind == dtype:
            if view.is_contiguous() and view.data_ptr() % 16 == 0:      # (elsewhere the sums have another order than in the copy)
                mine = view.clone()
                _run_distill(mine, k_, v_, temperature, t_, w_, kind, in_place=True)
                assert _same(mine, grad)
    return loss, stats


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("tailed", [False, True])
@pytest.mark.parametrize("rows,cols,k,temperature", [
    (1, 1, 1, 1.0), (2, 2, 1, 1.0), (3, 5, 3, 2.0), (4, 31, 31, 1.0), (7, 1000, 32, 0.5), (2, 1025, 1000, 1.5), (600, 260, 4, 1.0), (3, 50_257, 100, 2.0),
    (2, 128_003, 64, 1.0), (1, 262_144, 1024, 4.0), (5, 4_096, 7, 10.0)])
def test_distillation(dtype, tailed, rows, cols, k, temperature):
    rng = np.random.default_rng(cols + k)
    z = _logits(rng, rows, cols, dtype)
    keys, values = _teacher(rng, rows, cols, k, ragged=rows > 2)
    # (without any other class the student's rest is empty: a tail makes the loss infinite, which the edges below cover)
    tail = rng.uniform(0.01, 0.7, rows).astype(np.float32) if tailed and cols > k else None
    weight = np.where(rng.random(rows) < 0.8, rng.normal(0, 1, rows), 0.0).astype(np.float32) if rows > 2 else None
    _check_distill(z, dtype, keys, values, temperature, tail, weight)


@pytest.mark.parametrize("values_type", ["bf16", "fp16"])
def test_distillation_takes_the_teachers_values_in_any_type(values_type):
    rng = np.random.default_rng(2)
    z = _logits(rng, 4, 3_001, "bf16")
    keys, values = _teacher(rng, 4, 3_001, 17)
    _check_distill(z, "bf16", keys, values, 1.0, np.full(4, 0.2, np.float32), values_type=values_type)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("gap,shift", [(0, 1), (3, 0), (5, 7), (8, 8)])
@pytest.mark.parametrize("cols", [37, 5_003])
def test_distillation_of_rows_at_any_place(dtype, gap, shift, cols):
    rng = np.random.default_rng(cols + gap)
    z = _logits(rng, 5, cols, dtype)
    keys, values = _teacher(rng, 5, cols, 9)
    tail = np.full(5, 0.1, np.float32)
    store, view = _strided(z, dtype, gap, shift)
    _check_distill(z, dtype, keys, values, 1.0, tail, view=view)
    assert _untouched(store, view)
    # gradients at other places than the logits' (their rows begin at other elements), between values that stay
    k_, v_, t_ = _dev(keys), _dev(values), _dev(tail)
    for kind, g_gap, g_shift in itertools.product(dict.fromkeys([dtype, "fp32"]), (0, 2), (0, 1, 3)):
        _, want, _ = _run_distill(view, k_, v_, 1.0, t_, None, kind)
        g_store, grad = _strided(np.zeros((5, cols)), kind, g_gap, g_shift)
        assert binding.distill_loss(view, k_, v_, grad=grad, tail=t_) == 0
        assert torch.equal(grad, want) and _untouched(g_store, grad)
    _, want, _ = _run_distill(view, k_, v_, 1.0, t_, None, dtype)
    _run_distill(view, k_, v_, 1.0, t_, None, dtype, in_place=True)
    assert torch.equal(view, want) and _untouched(store, view)


def _edge(name, dtype):
    """(z, keys, values, temperature, tail, weight)"""
    rng = np.random.default_rng(3)
    rows, cols, k = 4, 2_003, 12
    z = _logits(rng, rows, cols, dtype)
    keys, values = _teacher(rng, rows, cols, k)
    t, tail, weight = 1.0, rng.uniform(0.05, 0.5, rows).astype(np.float32), None
    lowest = float(torch.finfo(TYPES[dtype]).min)
    if name == "no tail":
        tail = None
    elif name == "a tail of zero in some rows":
        tail[1:3] = 0.0
    elif name == "a tail of one":
        tail[1] = 1.0
    elif name == "pairs that are not there":
        keys[0, 1::2], keys[1, :], keys[2, :-1] = -1, cols, -5
    elif name == "repeated keys":
        keys[0, :] = keys[0, 0]
        keys[1, ::2] = keys[1, 0]
        keys[2, 5] = keys[2, 11]
    elif name == "repeated keys, no tail":
        keys[0, :] = keys[0, 0]
        keys[2, 5] = keys[2, 11]
        tail = None
    elif name == "padded rows of NaN":
        z[1], values[2], weight = np.nan, np.nan, np.array([1.0, 0.0, 0.0, 2.0])
    elif name == "pairs of no probability":
        values[0, :5], values[1, :] = -np.inf, -np.inf
    elif name == "ruled out classes":
        z[:, 100:1500] = -np.inf
        z[np.arange(rows)[:, None], keys] = 1.0
    elif name == "classes at the lowest value":
        z[:, 100:1500] = lowest
        z[np.arange(rows)[:, None], keys] = 1.0
    elif name == "rows at the lowest value":
        z[1] = lowest
    elif name == "keys that are ruled out":
        z[0, keys[0, 3]] = -np.inf
        values[1, 3] = -np.inf
        z[1, keys[1, 3]] = -np.inf
    elif name == "the rest ruled out":
        z[1] = -np.inf
        z[1, keys[1]] = 0.5
        z[2] = -np.inf
    elif name == "rows of -inf, no tail":
        z[1], tail = -np.inf, None
    elif name == "NaN":
        z[1, 7], values[2, 3] = np.nan, np.nan
    elif name == "a sure student":
        z[:] = np.clip(z, -3, 3)
        z[np.arange(rows), keys[:, 0]] = 60.0
        z[1, keys[1, 0]] = 90.0
    elif name == "a sure student elsewhere":
        z[:, 5] = 100.0
        keys[keys == 5] = 6
    elif name == "far logits":
        z += 30_000.0 if dtype == "fp16" else 1e6
        z = torch.from_numpy(z).to(TYPES[dtype]).double().numpy()
    elif name == "cold":
        t = 0.03
    elif name == "hot":
        t = 1000.0
    elif name == "all classes are keys":
        z, tail = z[:, :k].copy(), None
        keys = np.stack([rng.permutation(k) for _ in range(rows)]).astype(np.int32)
    return z, keys, values, t, tail, weight


EDGES = ["no tail", "a tail of zero in some rows", "a tail of one", "pairs that are not there", "repeated keys", "repeated keys, no tail", "padded rows of NaN",
         "pairs of no probability", "ruled out classes", "classes at the lowest value", "rows at the lowest value", "keys that are ruled out",
         "the rest ruled out", "rows of -inf, no tail", "NaN", "a sure student", "a sure student elsewhere", "far logits", "cold", "hot", "all classes are keys"]


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("name", EDGES)
def test_distillation_edges(dtype, name):
    z, keys, values, t, tail, weight = _edge(name, dtype)
    _check_distill(z, dtype, keys, values, t, tail, weight)


def test_distillation_slope_of_the_library_itself():
    """The gradient against differences of the loss, both from the library."""
    rng = np.random.default_rng(8)
    cols, t = 9, 2.0
    z0 = rng.normal(0, 1, cols)
    keys, values = np.array([[2, 5, 7]], np.int32), rng.normal(0, 1, (1, 3)).astype(np.float32)
    h = 2.0 ** -5
    z = np.stack([z0] + [z0 + s * h * np.eye(cols)[j] for j in range(cols) for s in (1, -1)]).astype(np.float32)
    rows = z.shape[0]
    loss, grad, _ = _run_distill(_dev(z), _dev(np.repeat(keys, rows, 0)), _dev(np.repeat(values, rows, 0)), t, torch.full((rows,), 0.25, device="cuda"), None, "fp32")
    loss, grad = loss.double().cpu().numpy(), grad.double().cpu().numpy()
    slope = (loss[1::2] - loss[2::2]) / (2 * h)
    # the third derivative is at most T^2 / T^3 = 1 / T in size, twice over; a loss of about 4 is off by some 2^-20
    assert np.all(np.abs(slope - grad[0]) <= h * h / 6 * 2 / t + 2.0 ** -20 * 4 / h)


def test_distillation_is_the_same_every_time_and_on_another_stream():
    rng = np.random.default_rng(9)
    z, (keys, values) = _dev(_logits(rng, 40, 30_011, "bf16"), torch.bfloat16), map(_dev, _teacher(rng, 40, 30_011, 50))
    tail = torch.full((40,), 0.3, device="cuda")
    first = _run_distill(z, keys, values, 1.0, tail, None, "bf16")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        second = _run_distill(z, keys, values, 1.0, tail, None, "bf16")
    side.synchronize()
    for a, b in zip(first, second):
        assert _same(a, b)
    # a caller's stream given by hand
    loss, alone = torch.empty(40, device="cuda"), _run_distill(z, keys, values, 1.0, tail, None, None)[0]
    side.wait_stream(torch.cuda.current_stream())
    assert binding.distill_loss(z, keys, values, loss=loss, tail=tail, stream=side) == 0
    side.synchronize()
    assert _same(loss, alone)


@pytest.mark.parametrize("cols", [60_001, 128_000])
def test_many_rows_of_several_blocks_beside_other_work(cols):
    """Rows that two and more blocks share, handed out as blocks become free: what runs beside them delays some blocks and not others."""
    rows, k = 3_001, 64
    gen = torch.Generator(device="cuda").manual_seed(cols)
    z = torch.randn((rows, cols), generator=gen, device="cuda").to(torch.bfloat16)
    keys = torch.randint(0, cols, (rows, k), generator=gen, device="cuda", dtype=torch.int32)
    values = torch.randn((rows, k), generator=gen, device="cuda")
    tail = torch.rand(rows, generator=gen, device="cuda") * 0.9
    side, other = torch.cuda.Stream(), torch.randn(3_000_000, device="cuda")
    first = None
    for turn in range(12):
        loss, grad = torch.full((rows,), MARK, device="cuda"), torch.empty_like(z)
        torch.cuda.synchronize()
        for _ in range(turn):
            with torch.cuda.stream(side):
                for n in (300, 3_000_000, 60_000):
                    other[:n] = other[:n] * 0.5 + 1.0
        assert binding.distill_loss(z, keys, values, loss=loss, grad=grad, tail=tail) == 0
        for _ in range(4 * turn):
            with torch.cuda.stream(side):
                for n in (60_000, 300, 3_000_000):
                    other[:n] = other[:n] * 0.5 + 1.0
        torch.cuda.synchronize()
        if first is None:
            first = loss, grad
        assert _same(loss, first[0]) and _same(grad, first[1])
    for r in (0, 1_500, rows - 1):
        want_loss, want_grad, grad_err, loss_err = ref.distill(z[r:r + 1].double().cpu().numpy(), keys[r:r + 1].cpu().numpy(), values[r:r + 1].double().cpu().numpy(), 1.0,
                                                               tail[r:r + 1].double().cpu().numpy())
        assert abs(loss[r].item() - want_loss[0]) <= loss_err[0]
        off = np.abs(grad[r].double().cpu().numpy() - want_grad[0])
        assert np.all(off <= grad_err[0] + ref.HALF_STEP["bf16"] * (np.abs(want_grad[0]) + grad_err[0]) + 2.0 ** -120)


def test_rows_beyond_two_to_the_31_elements():
    """Offsets of the last rows pass 32 bits: 2.2 G elements of bf16, gradient in place."""
    rows, cols, k = 17_200, 128_003, 5
    z = torch.empty((rows, cols), dtype=torch.bfloat16, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(1)
    block = torch.randn((400, cols), generator=gen, device="cuda").to(torch.bfloat16)
    for a in range(0, rows, 400):
        z[a:a + 400] = block
    keys, values, lse, tail = _run_top(z, k, 1.0)
    probe = [0, 399, 8_191, 16_776, 16_777, rows - 1]
    for r in probe:
        want_keys, want_values, _, _ = ref.top(z[r:r + 1].double().cpu().numpy(), k)
        assert np.array_equal(keys[r:r + 1].cpu().numpy(), want_keys)
    assert torch.equal(keys[16_800:17_200], keys[:400]) and _same(lse[16_800:17_200], lse[:400])
    values = values.float().flip(1).contiguous()
    want = {r: ref.distill(z[r:r + 1].double().cpu().numpy(), keys[r:r + 1].cpu().numpy(), values[r:r + 1].double().cpu().numpy(), 1.0, tail[r:r + 1].double().cpu().numpy())
            for r in probe}
    loss = torch.empty(rows, device="cuda")
    assert binding.distill_loss(z, keys, values, loss=loss, grad=z, tail=tail) == 0
    for r, (want_loss, want_grad, grad_err, loss_err) in want.items():
        assert abs(loss[r].item() - want_loss[0]) <= loss_err[0]
        off = np.abs(z[r].double().cpu().numpy() - want_grad[0])
        assert np.all(off <= grad_err[0] + ref.HALF_STEP["bf16"] * (np.abs(want_grad[0]) + grad_err[0]) + 2.0 ** -120)


# ---- the router's counts and balance loss -------------------------------------------------------------

def _workspace():
    binding.ensure_workspace(1, binding.params(1.1))


def _check_balance(rng, tokens, experts, k, dtype, segments=None, masked=False, coef=0.01, gap=0, shift=0, x=None, grad_types=None):
    _workspace()
    x = _logits(rng, tokens, experts, dtype) if x is None else x
    selected = np.argsort(-x, 1, kind="stable")[:, :k].astype(np.int32)
    if masked:
        selected[rng.random((tokens, k)) < 0.1] = -1
        selected[rng.random((tokens, k)) < 0.05] = experts
    mask = rng.random(tokens) < 0.8 if masked else None
    offsets = None if segments is None else np.asarray(segments, np.int64)
    n_seg = 1 if segments is None else len(segments) - 1
    want_counts, want_counted = ref.counts(selected, experts, mask, offsets)
    counts, counted = torch.full((n_seg, experts), -3, dtype=torch.int32, device="cuda"), torch.full((n_seg,), -3, dtype=torch.int32, device="cuda")
    m_, o_ = None if mask is None else _dev(mask), None if offsets is None else _dev(offsets)
    assert binding.expert_counts(_dev(selected), counts, counted, mask=m_, offsets=o_) == 0
    assert np.array_equal(counts.cpu().numpy(), want_counts) and np.array_equal(counted.cpu().numpy(), want_counted)
    up = rng.normal(0, 1, n_seg).astype(np.float32)
    store, view = _strided(x, dtype, gap, shift)
    for kind in grad_types or dict.fromkeys([dtype, "fp32"]):
        for gl in (None, up):
            want_loss, want_grad, grad_err, loss_err = ref.balance(x, want_counts, want_counted, coef, mask, offsets, gl)
            loss = torch.full((n_seg,), MARK, device="cuda")
            g_store, grad = _strided(np.full(x.shape, MARK), kind, gap, shift)
            assert binding.balance_loss(view, counts, counted, loss=loss, grad=grad, coef=coef, mask=m_, offsets=o_, grad_loss=None if gl is None else _dev(gl)) == 0
            got = grad.double().cpu().numpy()
            outside = np.isnan(want_grad)
            assert np.all(got[outside] == MARK) and _untouched(g_store, grad)
            tol = grad_err + ref.HALF_STEP[kind] * (np.abs(want_grad) + grad_err) + ref.LEAST[kind] + 2.0 ** -120
            assert np.all(np.abs(got - want_grad)[~outside] <= tol[~outside]), np.nanmax(np.abs(got - want_grad) - tol)
            # (the sum over the tokens is in fp64; one rounding at the end)
            assert np.all(np.abs(loss.double().cpu().numpy() - want_loss) <= loss_err + 2 * ref.U * np.abs(want_loss))
            again = torch.full_like(loss, MARK)
            assert binding.balance_loss(view, counts, counted, loss=again, coef=coef, mask=m_, offsets=o_) == 0 and _same(again, loss)
            alone = torch.full_like(grad, MARK)
            assert binding.balance_loss(view, counts, counted, grad=alone, coef=coef, mask=m_, offsets=o_, grad_loss=None if gl is None else _dev(gl)) == 0
            assert torch.equal(alone, grad)
    assert _untouched(store, view)
    if gap == 0 and shift == 0:
        assert binding.balance_loss(view, counts, counted, grad=view, coef=coef, mask=m_, offsets=o_) == 0       # in the logits' place
        other = torch.full_like(view, MARK)
        fresh = _dev(x, TYPES[dtype])
        assert binding.balance_loss(fresh, counts, counted, grad=other, coef=coef, mask=m_, offsets=o_) == 0
        outside = torch.from_numpy(np.isnan(ref.balance(x, want_counts, want_counted, coef, mask, offsets)[1])).cuda()
        assert torch.equal(view, torch.where(outside, fresh, other))


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("tokens,experts,k", [(1, 1, 1), (1, 8, 2), (64, 8, 2), (100, 3, 3), (777, 60, 6), (513, 64, 1), (301, 256, 8), (50, 257, 16), (40, 1000, 4), (33, 1024, 32)])
def test_balance_of_one_segment(dtype, tokens, experts, k):
    rng = np.random.default_rng(tokens + experts)
    _check_balance(rng, tokens, experts, k, dtype)
    _check_balance(rng, tokens, experts, k, dtype, masked=True, coef=-1.5)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("tokens,experts,k,segments", [
    (500, 16, 2, [0, 0, 7, 7, 300, 500, 500]), (500, 60, 4, [3, 100, 101, 499]), (6_000, 8, 2, list(range(0, 6_001, 5))), (90, 256, 8, [0, 90]), (40, 7, 1, [40, 40, 40])])
def test_balance_by_segments(dtype, tokens, experts, k, segments):
    rng = np.random.default_rng(tokens + experts)
    _check_balance(rng, tokens, experts, k, dtype, segments)
    _check_balance(rng, tokens, experts, k, dtype, segments, masked=True)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("gap,shift,experts", [(0, 1, 40), (4, 0, 60), (3, 5, 256), (8, 8, 128), (1, 0, 7)])
def test_balance_of_rows_at_any_place(dtype, gap, shift, experts):
    _check_balance(np.random.default_rng(gap), 70, experts, 3, dtype, [0, 30, 66], True, gap=gap, shift=shift)


@pytest.mark.parametrize("dtype", list(TYPES))
def test_balance_edges(dtype):
    rng = np.random.default_rng(4)
    x = _logits(rng, 60, 24, dtype)
    x[3], x[4, 5:], x[5], x[6, 2] = -np.inf, -np.inf, float(torch.finfo(TYPES[dtype]).min), 200.0
    _check_balance(rng, 60, 24, 2, dtype, x=x)
    # tokens that do not count may hold anything; no token that counts; no selection at all
    _workspace()
    x[:] = np.nan
    x[:10] = 0.5
    view = _dev(x, TYPES[dtype])
    mask = torch.zeros(60, dtype=torch.bool, device="cuda")
    mask[:10] = True
    counts, counted = torch.ones((1, 24), dtype=torch.int32, device="cuda"), torch.full((1,), 10, dtype=torch.int32, device="cuda")
    loss, grad = torch.empty(1, device="cuda"), torch.empty_like(view)
    assert binding.balance_loss(view, counts, counted, loss=loss, grad=grad, mask=mask) == 0
    assert abs(loss.item() - 1.0) < 1e-6 and torch.equal(grad[10:], torch.zeros_like(grad[10:]))
    for c, n in ((counts, counted * 0), (counts * 0, counted)):
        assert binding.balance_loss(view, c, n, loss=loss, grad=grad, mask=mask) == 0
        assert loss.item() == 0.0 and not grad.any()
    # no tokens
    none = view[:0]
    assert binding.expert_counts(torch.empty((0, 2), dtype=torch.int32, device="cuda"), counts, counted) == 0
    assert not counts.any() and not counted.any()
    assert binding.balance_loss(none, counts, counted, loss=loss, grad=grad[:0]) == 0 and loss.item() == 0.0


def test_balance_needs_its_workspace():
    small = torch.zeros(binding.debug_layout()["queue_slots"] + (4 << 17) + (8 << 17) + 8 * 2048, dtype=torch.uint8, device="cuda")      # its fixed part and no segment
    binding.set_workspace(small)
    x, counts, counted = torch.zeros(4, 8, device="cuda"), torch.ones((1, 8), dtype=torch.int32, device="cuda"), torch.full((1,), 4, dtype=torch.int32, device="cuda")
    loss = torch.empty(1, device="cuda")
    assert binding.balance_loss(x, counts, counted, loss=loss) == binding.E_NO_WORKSPACE
    assert binding.balance_loss(x, counts, counted, grad=torch.empty_like(x)) == 0          # (the gradient alone needs none)
    torch.cuda.synchronize()
    _workspace()
    assert binding.balance_loss(x, counts, counted, loss=loss) == 0 and abs(loss.item() - 1.0) < 1e-6


def test_counts_of_many_tokens():
    rng = np.random.default_rng(12)
    tokens, k, experts = 200_003, 5, 100
    selected = rng.integers(-1, experts + 1, (tokens, k)).astype(np.int32)
    selected[:, 0] = 17                                                        # everybody's favourite
    mask = rng.random(tokens) < 0.5
    counts, counted = torch.empty((1, experts), dtype=torch.int32, device="cuda"), torch.empty((1,), dtype=torch.int32, device="cuda")
    assert binding.expert_counts(_dev(selected), counts, counted, mask=_dev(mask)) == 0
    kept = selected[mask]
    want = np.bincount(kept[(kept >= 0) & (kept < experts)].ravel(), minlength=experts)
    assert np.array_equal(counts[0].cpu().numpy(), want) and counted.item() == mask.sum()


# ---- together -----------------------------------------------------------------------------------------

def test_binding_refuses_what_the_library_cannot_see():
    z, keys, values = torch.zeros(4, 64, device="cuda"), torch.zeros((4, 3), dtype=torch.int32, device="cuda"), torch.zeros(4, 3, device="cuda")
    loss = torch.empty(4, device="cuda")
    for bad in (dict(student=z.t()), dict(student=z.double()), dict(keys=keys.long()), dict(keys=keys.cpu()), dict(values=values[:3]), dict(loss=loss[:3]),
                dict(loss=loss.double()), dict(grad=z.cpu()), dict(tail=loss[:2]), dict(stats=loss), dict(keys=keys.t().contiguous().t())):
        with pytest.raises(AssertionError):
            binding.distill_loss(**{**dict(student=z, keys=keys, values=values, loss=loss), **bad})
    assert binding.distill_loss(z.expand(4, 64)[:1].expand(4, 64), keys, values, loss=loss) == binding.E_BAD_PARAM      # (rows on top of one another)
    with pytest.raises(AssertionError):
        binding.balance_loss(z, torch.zeros((2, 64), dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda"), loss=loss[:2])
    with pytest.raises(AssertionError):
        binding.top_logits(z, keys, values.half())


def _step(student_w, x, router_w, teacher, selected, coef):
    """A worker's step: losses of a linear student and its router, and the gradient of both weights as one vector."""
    keys, values, tail = teacher
    rows = x.shape[0]
    z, gates = x @ student_w.t(), x @ router_w.t()
    loss, dz = torch.empty(rows, device="cuda"), torch.empty_like(z)
    weight = torch.full((rows,), 1.0 / rows, device="cuda")
    assert binding.distill_loss(z, keys, values, loss=loss, grad=dz, temperature=2.0, tail=tail, weight=weight) == 0
    counts, counted = torch.empty((1, router_w.shape[0]), dtype=torch.int32, device="cuda"), torch.empty(1, dtype=torch.int32, device="cuda")
    picked = torch.empty((rows, selected), dtype=torch.int32, device="cuda")
    assert binding.top_logits(gates, picked, torch.empty((rows, selected), device="cuda")) == 0
    assert binding.expert_counts(picked, counts, counted) == 0
    balance, dg = torch.empty(1, device="cuda"), torch.empty_like(gates)
    assert binding.balance_loss(gates, counts, counted, loss=balance, grad=dg, coef=coef) == 0
    return loss.sum() + balance[0], torch.cat([(dz.t() @ x).reshape(-1), (dg.t() @ x).reshape(-1)]), (z, gates, counts, counted)


def test_a_workers_step_from_the_losses_to_the_update():
    """Teacher's top logits -> losses and gradients of two workers -> streams -> one Adam step, and the gradient of it all."""
    torch.backends.cuda.matmul.allow_tf32 = False
    gen = torch.Generator(device="cuda").manual_seed(3)
    vocab, experts, width, rows, k = 1_003, 12, 32, 96, 20
    n = (vocab + experts) * width
    p = binding.params(1.1)
    binding.ensure_workspace(n, p)
    teacher_w = torch.randn((vocab, width), generator=gen, device="cuda")
    theta = 0.1 * torch.randn(n, generator=gen, device="cuda")
    m, v, scratch = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    x = torch.randn((2, rows, width), generator=gen, device="cuda")
    split = vocab * width
    streams, sizes, grads = [], [], []
    for w in range(2):
        keys, values = torch.empty((rows, k), dtype=torch.int32, device="cuda"), torch.empty((rows, k), device="cuda")
        tail = torch.empty(rows, device="cuda")
        assert binding.top_logits(x[w] @ teacher_w.t(), keys, values, temperature=2.0, tail=tail) == 0
        total, grad, (z, gates, counts, counted) = _step(theta[:split].view(vocab, width), x[w], theta[split:].view(experts, width), (keys, values, tail), 3, 0.5)
        # the whole gradient against the formulas' in 64 bits
        _, dz, dz_err, _ = ref.distill(z.double().cpu().numpy(), keys.cpu().numpy(), values.double().cpu().numpy(), 2.0, tail.double().cpu().numpy(), np.full(rows, 1.0 / rows))
        _, dg, dg_err, _ = ref.balance(gates.double().cpu().numpy(), counts.cpu().numpy(), counted.cpu().numpy(), 0.5)
        x64 = x[w].double().cpu().numpy()
        want = np.concatenate([(dz.T @ x64).ravel(), (dg.T @ x64).ravel()])
        size = np.concatenate([(np.abs(dz).T @ np.abs(x64)).ravel(), (np.abs(dg).T @ np.abs(x64)).ravel()])
        err = np.concatenate([((dz_err + ref.U * np.abs(dz)).T @ np.abs(x64)).ravel(), ((dg_err + ref.U * np.abs(dg)).T @ np.abs(x64)).ravel()])
        assert np.all(np.abs(grad.double().cpu().numpy() - want) <= err + rows * ref.U * size + 1e-30)      # (a product over `rows` terms in fp32)
        out = torch.zeros(binding.compress_bound(n, p), dtype=torch.uint8, device="cuda")
        assert binding.compress(grad, p, out) == 0
        size_, kept, status = binding.stream_info(out)
        assert status == 0 and kept > 0
        streams.append(out)
        sizes.append(size_)
        grads.append(grad)
        assert torch.isfinite(total)
    before = theta.clone()
    assert binding.sparse_adam_update_batch(streams, sizes, n, p, binding.Adam(0.01, 0.9, 0.999, 1e-8), scratch, theta, m, v) == 0
    assert binding.decode_status() == 0
    moved = theta != before
    # the step goes against the decoded gradient, which has the workers' signs
    dense = torch.zeros(n, device="cuda")
    assert binding.decompress_accumulate_batch(streams, sizes, n, p, dense) == 0 and binding.decode_status() == 0
    assert torch.equal(moved, dense != 0) and bool(((theta - before).sign() == -dense.sign())[moved].all())


def test_a_step_captured_and_replayed():
    gen = torch.Generator(device="cuda").manual_seed(4)
    vocab, experts, width, rows = 2_000, 16, 24, 64
    _workspace()
    student, router = torch.randn((vocab, width), generator=gen, device="cuda"), torch.randn((experts, width), generator=gen, device="cuda")
    x = torch.randn((rows, width), generator=gen, device="cuda")
    z, gates = x @ student.t(), x @ router.t()
    keys, values, tail = torch.empty((rows, 8), dtype=torch.int32, device="cuda"), torch.empty((rows, 8), device="cuda"), torch.empty(rows, device="cuda")
    loss, dz, stats, back = torch.empty(rows, device="cuda"), torch.empty_like(z), torch.empty((rows, 2), device="cuda"), torch.empty_like(z)
    picked, picked_v = torch.empty((rows, 2), dtype=torch.int32, device="cuda"), torch.empty((rows, 2), device="cuda")
    counts, counted = torch.empty((1, experts), dtype=torch.int32, device="cuda"), torch.empty(1, dtype=torch.int32, device="cuda")
    balance, dg = torch.empty(1, device="cuda"), torch.empty_like(gates)
    outs = [keys, values, tail, loss, dz, stats, back, picked, picked_v, counts, counted, balance, dg]

    def step():
        assert binding.top_logits(z, keys, values, tail=tail) == 0
        assert binding.distill_loss(z, keys, values, loss=loss, grad=dz, stats=stats, temperature=3.0, tail=tail) == 0
        assert binding.distill_loss_backward(z, keys, values, stats, back, temperature=3.0, tail=tail) == 0
        assert binding.top_logits(gates, picked, picked_v) == 0
        assert binding.expert_counts(picked, counts, counted) == 0
        assert binding.balance_loss(gates, counts, counted, loss=balance, grad=dg) == 0

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    for seed in (5, 6):
        z.copy_(torch.randn(z.shape, generator=gen.manual_seed(seed), device="cuda"))
        gates.copy_(torch.randn(gates.shape, generator=gen, device="cuda"))
        step()
        torch.cuda.synchronize()
        want = [o.clone() for o in outs]
        for o in outs:
            o.fill_(1)
        graph.replay()
        graph.replay()
        torch.cuda.synchronize()
        for o, w in zip(outs, want):
            assert _same(o, w)
