"""The losses on logits without a GPU: the 64-bit forms against the definition's own properties and differences, and what the
library's entry points refuse before any launch."""
import ctypes as C

import numpy as np
import pytest

import loss_ref as ref
from paper_2112_04291_b200 import binding, build

FAKE = 1 << 20        # never dereferenced: the checks fail before any launch


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.lib()


def _pairs(rng, rows, cols, k, repeat=False):
    keys = np.stack([rng.choice(cols, k, replace=repeat) for _ in range(rows)])
    return keys, rng.normal(0, 2, (rows, k))


# ---- the 64-bit forms ----------------------------------------------------------------------------

@pytest.mark.parametrize("tailed", [False, True])
@pytest.mark.parametrize("repeat", [False, True])
def test_distillation_gradient_is_the_losss_slope(tailed, repeat):
    rng = np.random.default_rng(5)
    rows, cols, k, t = 3, 23, 6, 1.7
    z = rng.normal(0, 2, (rows, cols))
    keys, values = _pairs(rng, rows, cols, k, repeat)
    keys[1, 2] = -1
    tail = rng.uniform(0.05, 0.6, rows) if tailed else None
    weight = np.array([1.0, 0.5, -2.0])
    _, grad, _, _ = ref.distill(z, keys, values, t, tail, weight)
    h = 1e-5
    for j in range(cols):
        up, down = z.copy(), z.copy()
        up[:, j] += h
        down[:, j] -= h
        slope = (ref.distill(up, keys, values, t, tail, weight)[0] - ref.distill(down, keys, values, t, tail, weight)[0]) / (2 * h)
        # central differences: h^2 / 6 of the third derivative (at most about 2 T w) and rounding 2^-52 |loss| / h
        assert np.all(np.abs(slope - grad[:, j]) < 1e-9 + 2.0 ** -50 * 50 / h)
    # (without repeated keys the classes' gradients cancel: the loss does not change when all logits move together)
    assert np.all(np.abs(grad.sum(1)) < 1e-12)


def test_distillation_is_zero_where_the_student_agrees_with_the_teacher():
    rng = np.random.default_rng(6)
    z = rng.normal(0, 2, (4, 40))
    keys, values, _, tail = ref.top(z, 7, 2.0)
    loss, grad, _, _ = ref.distill(z, keys, values, 2.0, tail)
    # the pairs and the tail are the student's own: no divergence, and a gradient of zero
    assert np.all(np.abs(loss) < 1e-14) and np.all(np.abs(grad) < 1e-14)
    whole = ref.distill(z, np.tile(np.arange(40), (4, 1)), z, 2.0)
    assert np.all(np.abs(whole[0]) < 1e-14) and np.all(np.abs(whole[1]) < 1e-14)


def test_balance_gradient_is_the_losss_slope_and_a_uniform_router_has_loss_coef():
    rng = np.random.default_rng(7)
    x = rng.normal(0, 1, (11, 6))
    selected = np.argsort(-x, 1)[:, :2]
    mask = rng.random(11) < 0.7
    offsets = [1, 4, 4, 10]
    count, counted = ref.counts(selected, 6, mask, offsets)
    gl = np.array([0.5, 1.0, -2.0])
    _, grad, _, _ = ref.balance(x, count, counted, 0.3, mask, offsets, gl)
    h = 1e-5
    for e in range(6):
        for t in range(1, 10):
            up, down = x.copy(), x.copy()
            up[t, e] += h
            down[t, e] -= h
            slope = (gl * (ref.balance(up, count, counted, 0.3, mask, offsets)[0] - ref.balance(down, count, counted, 0.3, mask, offsets)[0])).sum() / (2 * h)
            assert abs(slope - grad[t, e]) < 1e-9
    flat = ref.balance(np.zeros((8, 4)), np.full((1, 4), 4), np.array([8]), 0.7)
    assert abs(flat[0][0] - 0.7) < 1e-15 and np.all(flat[1] == 0)
    # the parts of two workers that share their counts add up to the loss of all their tokens
    both = ref.balance(x, *ref.counts(selected, 6), 0.3)[0]
    parts = [ref.balance(x[a:b], *ref.counts(selected, 6), 0.3)[0] for a, b in ((0, 5), (5, 11))]
    assert abs(both - sum(parts)) < 1e-15


def test_top_orders_ties_and_nan_as_stated():
    z = np.array([[1.0, np.nan, 3.0, 3.0, -0.0, 0.0, -np.inf, np.inf]])
    keys, _, lse, tail = ref.top(z, 8)
    assert keys.tolist() == [[1, 7, 2, 3, 0, 4, 5, 6]] and np.isnan(lse[0]) and np.isnan(tail[0])


# ---- refusals -------------------------------------------------------------------------------------

def _matrix(**changes):
    m = dict(data=FAKE, rows=4, cols=100, row_stride=100, type=binding.F32, reserved=0)
    m.update(changes)
    return binding.Matrix(*[m[n] for n, _ in binding.Matrix._fields_])


def _teacher(**changes):
    m = dict(keys=FAKE, values=FAKE, tail=None, k=4, type=binding.F32)
    m.update(changes)
    return binding.Pairs(*[m[n] for n, _ in binding.Pairs._fields_])


BAD_MATRICES = [
    (dict(type=3), "E_BAD_PARAM"), (dict(reserved=1), "E_BAD_PARAM"), (dict(row_stride=99), "E_BAD_PARAM"), (dict(row_stride=0), "E_BAD_PARAM"),
    (dict(row_stride=1 << 31), "E_BAD_PARAM"), (dict(cols=0), "E_BAD_N"), (dict(cols=1 << 31, row_stride=1 << 31), "E_BAD_N"), (dict(rows=1 << 31), "E_BAD_N"),
    (dict(data=None), "E_NULL"), (dict(data=FAKE + 2), "E_ALIGN"), (dict(type=binding.BF16, data=FAKE + 1), "E_ALIGN"),
]


@pytest.mark.parametrize("changes,code", BAD_MATRICES)
def test_matrices_that_every_entry_refuses(lib, changes, code):
    bad, good, t, code = _matrix(**changes), _matrix(), _teacher(), getattr(binding, code)
    ref_ = C.byref
    assert lib.fastsgd_top_logits(ref_(bad), 4, 1.0, FAKE, FAKE, None, None, None) == code
    assert lib.fastsgd_distill_loss(ref_(bad), ref_(t), 1.0, None, FAKE, None, None, None) == code
    assert lib.fastsgd_balance_loss(ref_(bad), None, None, 1, FAKE, FAKE, 1.0, None, FAKE, None, None) == code
    far = _matrix(**{"data": FAKE + (1 << 16), **changes})      # (a gradient)
    if changes.get("data", 1) is not None and "data" not in changes:
        assert lib.fastsgd_distill_loss(ref_(good), ref_(t), 1.0, None, FAKE, None, ref_(far), None) == code
        assert lib.fastsgd_distill_loss_backward(ref_(good), ref_(t), 1.0, None, FAKE, None, ref_(far), None) == code
        assert lib.fastsgd_balance_loss(ref_(good), None, None, 1, FAKE, FAKE, 1.0, None, None, ref_(far), None) == code


def test_top_logits_refusals(lib):
    m = C.byref(_matrix())
    call = lib.fastsgd_top_logits
    assert call(None, 4, 1.0, FAKE, FAKE, None, None, None) == binding.E_NULL
    assert call(m, 4, 1.0, None, FAKE, None, None, None) == binding.E_NULL
    assert call(m, 4, 1.0, FAKE, None, None, None, None) == binding.E_NULL
    for k in (0, 101, 1025):
        assert call(m, k, 1.0, FAKE, FAKE, None, None, None) == binding.E_BAD_PARAM
    for t in (0.0, -1.0, float("nan"), float("inf"), 1e-9, 1e9):
        assert call(m, 4, t, FAKE, FAKE, None, None, None) == binding.E_BAD_PARAM
    for args in ((FAKE + 1, FAKE, None, None), (FAKE, FAKE + 2, None, None), (FAKE, FAKE, FAKE + 1, None), (FAKE, FAKE, None, FAKE + 2)):
        assert call(m, 4, 1.0, *args, None) == binding.E_ALIGN
    wide = C.byref(_matrix(cols=(1 << 20) + 1, row_stride=(1 << 20) + 1))
    assert call(wide, 4, 1.0, FAKE, FAKE, None, None, None) == binding.E_NOT_IMPLEMENTED
    assert call(C.byref(_matrix(rows=0, data=None)), 4, 1.0, None, None, None, None, None) == binding.OK


def test_distillation_refusals(lib):
    m, t = C.byref(_matrix()), C.byref(_teacher())
    call, back = lib.fastsgd_distill_loss, lib.fastsgd_distill_loss_backward
    far = FAKE + (1 << 16)
    assert call(m, t, 1.0, None, None, None, None, None) == binding.E_NULL                 # nothing to write
    assert call(m, None, 1.0, None, FAKE, None, None, None) == binding.E_NULL
    assert call(m, C.byref(_teacher(keys=None)), 1.0, None, FAKE, None, None, None) == binding.E_NULL
    assert call(m, C.byref(_teacher(values=None)), 1.0, None, FAKE, None, None, None) == binding.E_NULL
    for changes in (dict(k=0), dict(k=1025), dict(type=7)):
        assert call(m, C.byref(_teacher(**changes)), 1.0, None, FAKE, None, None, None) == binding.E_BAD_PARAM
    for temp in (0.0, -1.0, float("nan"), float("inf")):
        assert call(m, t, temp, None, FAKE, None, None, None) == binding.E_BAD_PARAM
    for changes in (dict(keys=FAKE + 2), dict(values=FAKE + 2), dict(tail=FAKE + 1)):
        assert call(m, C.byref(_teacher(**changes)), 1.0, None, FAKE, None, None, None) == binding.E_ALIGN
    assert call(m, t, 1.0, FAKE + 1, FAKE, None, None, None) == binding.E_ALIGN
    wide = C.byref(_matrix(cols=(1 << 20) + 1, row_stride=(1 << 20) + 1))
    assert call(wide, t, 1.0, None, FAKE, None, None, None) == binding.E_NOT_IMPLEMENTED
    # gradients of another shape or type, or that overlap the logits without being in their place
    for changes in (dict(rows=5), dict(cols=99), dict(type=binding.F16)):
        assert call(m, t, 1.0, None, FAKE, None, C.byref(_matrix(**{"data": far, **changes})), None) == binding.E_BAD_PARAM
    for changes in (dict(data=FAKE + 400), dict(row_stride=128), dict(data=FAKE - 4)):
        assert call(m, t, 1.0, None, FAKE, None, C.byref(_matrix(**changes)), None) == binding.E_BAD_PARAM
    half = C.byref(_matrix(type=binding.BF16))
    assert call(half, t, 1.0, None, FAKE, None, m, None) == binding.E_BAD_PARAM            # fp32 over 16-bit logits
    assert back(m, t, 1.0, None, FAKE, None, None, None) == binding.E_NULL
    assert back(m, t, 1.0, None, None, None, C.byref(_matrix(data=far)), None) == binding.E_NULL
    none = C.byref(_matrix(rows=0, data=None))
    assert call(none, C.byref(_teacher(keys=None, values=None)), 1.0, None, FAKE, None, None, None) == binding.OK
    assert back(none, C.byref(_teacher(keys=None, values=None)), 1.0, None, None, None, none, None) == binding.OK


def test_router_refusals(lib):
    count, loss = lib.fastsgd_expert_counts, lib.fastsgd_balance_loss
    assert count(FAKE, 4, 2, 0, None, None, 1, FAKE, FAKE, None) == binding.E_BAD_PARAM
    assert count(FAKE, 4, 2, 1025, None, None, 1, FAKE, FAKE, None) == binding.E_BAD_PARAM
    assert count(FAKE, 4, 0, 8, None, None, 1, FAKE, FAKE, None) == binding.E_BAD_PARAM
    assert count(FAKE, 4, 9, 8, None, None, 1, FAKE, FAKE, None) == binding.E_BAD_PARAM
    assert count(FAKE, 4, 2, 8, None, None, 0, FAKE, FAKE, None) == binding.E_BAD_PARAM
    assert count(FAKE, 4, 2, 8, None, FAKE, (1 << 24) + 1, FAKE, FAKE, None) == binding.E_BAD_PARAM
    assert count(FAKE, 4, 2, 8, None, None, 2, FAKE, FAKE, None) == binding.E_NULL         # several segments without offsets
    assert count(FAKE, 4, 2, 8, None, FAKE + 4, 2, FAKE, FAKE, None) == binding.E_ALIGN
    assert count(FAKE, 1 << 31, 2, 8, None, None, 1, FAKE, FAKE, None) == binding.E_BAD_N
    assert count(FAKE, 1 << 30, 4, 8, None, None, 1, FAKE, FAKE, None) == binding.E_BAD_N
    for args in ((None, FAKE, FAKE), (FAKE, None, FAKE), (FAKE, FAKE, None)):
        assert count(args[0], 4, 2, 8, None, None, 1, args[1], args[2], None) == binding.E_NULL
    for args in ((FAKE + 2, FAKE, FAKE), (FAKE, FAKE + 1, FAKE), (FAKE, FAKE, FAKE + 2)):
        assert count(args[0], 4, 2, 8, None, None, 1, args[1], args[2], None) == binding.E_ALIGN
    m, far = C.byref(_matrix()), FAKE + (1 << 16)
    assert loss(m, None, None, 1, FAKE, FAKE, 1.0, None, None, None, None) == binding.E_NULL
    assert loss(m, None, None, 1, None, FAKE, 1.0, None, FAKE, None, None) == binding.E_NULL
    assert loss(m, None, None, 1, FAKE, None, 1.0, None, FAKE, None, None) == binding.E_NULL
    assert loss(m, None, None, 2, FAKE, FAKE, 1.0, None, FAKE, None, None) == binding.E_NULL
    assert loss(m, None, None, 0, FAKE, FAKE, 1.0, None, FAKE, None, None) == binding.E_BAD_PARAM
    assert loss(m, None, None, 1, FAKE, FAKE, float("inf"), None, FAKE, None, None) == binding.E_BAD_PARAM
    assert loss(m, None, None, 1, FAKE, FAKE, 1.0, FAKE + 2, FAKE, None, None) == binding.E_ALIGN
    assert loss(C.byref(_matrix(cols=1025, row_stride=1025)), None, None, 1, FAKE, FAKE, 1.0, None, FAKE, None, None) == binding.E_BAD_PARAM
    assert loss(m, None, None, 1, FAKE, FAKE, 1.0, None, None, C.byref(_matrix(data=far, cols=99)), None) == binding.E_BAD_PARAM
    assert loss(m, None, None, 1, FAKE, FAKE, 1.0, None, None, C.byref(_matrix(data=FAKE + 4)), None) == binding.E_BAD_PARAM
