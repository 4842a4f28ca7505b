"""Operators on rows chosen by an id without a GPU: the definitions against differences, and what the entries refuse (nothing is launched)."""
import ctypes as C

import numpy as np
import pytest

import rows_ref as ref
from paper_2112_04291_b200 import binding, build

FAKE = 1 << 20      # never dereferenced: the checks fail before any launch


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.lib()


def test_order_puts_equal_ids_in_the_order_of_their_positions_and_leaves_others_out():
    order, starts, distinct = ref.order_ids(np.array([3, -1, 0, 3, 5, 0, 9]), 6)
    assert order.tolist() == [2, 5, 0, 3, 4] and starts.tolist() == [0, 2, 2, 2, 4, 4, 5] and distinct.tolist() == [0, 3, 5]


def test_gradients_are_the_slopes_of_the_forward_operators():
    """Both operators are linear in what the gradient is of: differences with a step of 1 are exact up to rounding."""
    rng = np.random.default_rng(1)
    ids = np.array([2, 0, 2, -1, 1, 2])
    table, up = rng.normal(size=(4, 3)), rng.normal(size=(6, 3))
    grad, _, _ = ref.embedding_backward(up, ids, 4, 0.7)
    for v, c in np.ndindex(4, 3):
        step = np.zeros((4, 3))
        step[v, c] = 1.0
        slope = (up * (ref.embedding(table + step, ids, 0.7) - ref.embedding(table, ids, 0.7))).sum()
        assert abs(slope - grad[v, c]) < 1e-12
    selected = np.array([[0, 2], [2, -1], [0, 1]])
    order, starts, _ = ref.order_ids(selected, 3)
    source = order // 2
    x, w = rng.normal(size=(3, 4)), rng.normal(size=(3, 5, 4))
    gy = rng.normal(size=(len(order), 5))
    gx, _ = ref.products_input(gy, starts, w)
    gw, _ = ref.products_weights(gy, x, source, starts)
    sum_gx, _, _ = ref.embedding_backward(gx, source, 3, 1.0)                # a token's gradient: the sum of its rows'

    def value(x, w):
        return (gy * ref.products(x, source, starts, w)[0]).sum()
    for i in np.ndindex(3, 4):
        step = np.zeros((3, 4))
        step[i] = 1.0
        assert abs(value(x + step, w) - value(x, w) - sum_gx[i]) < 1e-12
    for i in np.ndindex(3, 5, 4):
        step = np.zeros((3, 5, 4))
        step[i] = 1.0
        assert abs(value(x, w + step) - value(x, w) - gw[i]) < 1e-12


def _matrix(**changes):
    fields = dict(data=FAKE, rows=10, cols=16, row_stride=16, type=binding.BF16, reserved=0)
    fields.update(changes)
    return binding.Matrix(*fields.values())


def _experts(**changes):
    fields = dict(data=FAKE + (1 << 24), experts=4, outs=24, ins=16, row_stride=16, expert_stride=24 * 16, type=binding.BF16, reserved=0)
    fields.update(changes)
    return binding.Experts(*fields.values())


def test_workspace_sizes(lib):
    assert lib.fastsgd_rows_workspace_bytes(1 << 31, 1) == 0 and lib.fastsgd_rows_workspace_bytes(5, 0) == 0 and lib.fastsgd_rows_workspace_bytes(5, 1 << 31) == 0
    for count in (0, 1, 1000, 65_536, 65_537, 1 << 20, (1 << 31) - 1):
        for cols in (1, 8, 300, 4096, 20_000):
            need = lib.fastsgd_rows_workspace_bytes(count, cols)
            assert need >= 1 << 20 and need % 256 == 0
            if count > 65_536:
                assert need >= 16 * count


def test_order_refusals(lib):
    def call(ids=FAKE, count=10, span=5, order=FAKE, starts=FAKE, distinct=None, number=None):
        return lib.fastsgd_order_ids(ids, count, span, order, starts, distinct, number, None)
    assert call(ids=None) == binding.E_NULL and call(order=None) == binding.E_NULL and call(starts=None) == binding.E_NULL
    assert call(count=1 << 31) == binding.E_BAD_N and call(span=0) == binding.E_BAD_PARAM and call(span=(1 << 20) + 1) == binding.E_NOT_IMPLEMENTED
    for name in ("ids", "order", "starts", "distinct", "number"):
        assert call(**{name: FAKE + 2}) == binding.E_ALIGN


def test_embedding_refusals(lib):
    far = FAKE + (1 << 24)

    def lookup(table=_matrix(), ids=FAKE, out=_matrix(data=far)):
        return lib.fastsgd_embedding(table, ids, 1.0, out, None)

    def backward(grad=_matrix(), ids=FAKE, order=FAKE, starts=FAKE, out=_matrix(data=far)):
        return lib.fastsgd_embedding_backward(grad, ids, order, starts, 1.0, out, None)

    def pairs(grad=_matrix(), ids=FAKE, order=FAKE, starts=FAKE, distinct=FAKE, number=FAKE, span=100, keys=far, values=far + (1 << 24), most=10):
        return lib.fastsgd_embedding_backward_pairs(grad, ids, order, starts, distinct, number, span, 1.0, keys, values, most, None)
    assert lookup(table=None) == binding.E_NULL and lookup(ids=None) == binding.E_NULL and lookup(out=None) == binding.E_NULL and lookup(ids=FAKE + 1) == binding.E_ALIGN
    assert lookup(out=_matrix(data=far, cols=8)) == binding.E_BAD_PARAM and lookup(out=_matrix(data=far, type=binding.F16)) == binding.E_BAD_PARAM
    assert lookup(out=_matrix(data=FAKE + 64)) == binding.E_BAD_PARAM and lookup(out=_matrix(data=far, type=9)) == binding.E_BAD_PARAM
    assert lookup(table=_matrix(row_stride=15)) == binding.E_BAD_PARAM and lookup(table=_matrix(data=FAKE + 1)) == binding.E_ALIGN
    for name in ("grad", "ids", "order", "starts", "out"):
        assert backward(**{name: None}) == binding.E_NULL
    for name in ("ids", "order", "starts"):
        assert backward(**{name: FAKE + 2}) == binding.E_ALIGN
    assert backward(out=_matrix(data=far, cols=8)) == binding.E_BAD_PARAM and backward(out=_matrix(data=far, type=binding.F16)) == binding.E_BAD_PARAM
    assert backward(out=_matrix()) == binding.E_BAD_PARAM and backward(out=_matrix(data=None, rows=0)) == binding.E_BAD_N
    for name in ("grad", "ids", "order", "starts", "distinct", "number", "keys", "values"):
        assert pairs(**{name: None}) == binding.E_NULL
    for name in ("ids", "order", "starts", "distinct", "number", "keys", "values"):
        assert pairs(**{name: FAKE + 2}) == binding.E_ALIGN
    assert pairs(span=0) == binding.E_BAD_N and pairs(span=1 << 27) == binding.E_BAD_N and pairs(most=1 << 31) == binding.E_BAD_N
    assert pairs(span=1 << 60) == binding.E_BAD_N
    assert pairs(values=far) == binding.E_BAD_PARAM and pairs(keys=FAKE + 16) == binding.E_BAD_PARAM


def test_product_refusals(lib):
    far = FAKE + (1 << 25)
    x, w, y = _matrix(), _experts(), _matrix(data=far, rows=20, cols=24, row_stride=24)

    def forward(x=x, order=FAKE, per_row=2, starts=FAKE, w=w, y=y):
        return lib.fastsgd_expert_product(x, order, per_row, starts, w, y, None)

    def back_input(gy=y, starts=FAKE, w=w, gx=_matrix(rows=20)):
        return lib.fastsgd_expert_product_backward_input(gy, starts, w, gx, None)

    def back_weights(gy=y, x=x, order=FAKE, per_row=2, starts=FAKE, w=w):
        return lib.fastsgd_expert_product_backward_weights(gy, x, order, per_row, starts, w, None)
    for name in ("x", "starts", "w", "y"):
        assert forward(**{name: None}) == binding.E_NULL
    for name in ("gy", "starts", "w", "gx"):
        assert back_input(**{name: None}) == binding.E_NULL
    for name in ("gy", "x", "starts", "w"):
        assert back_weights(**{name: None}) == binding.E_NULL
    bad = [(dict(data=None), binding.E_NULL), (dict(experts=0), binding.E_BAD_PARAM), (dict(experts=1025), binding.E_BAD_PARAM), (dict(outs=0), binding.E_BAD_N), (dict(ins=1 << 31), binding.E_BAD_N),
           (dict(row_stride=8), binding.E_BAD_PARAM), (dict(expert_stride=24 * 16 - 8), binding.E_BAD_PARAM), (dict(type=7), binding.E_BAD_PARAM), (dict(reserved=1), binding.E_BAD_PARAM),
           (dict(data=FAKE + (1 << 24) + 8), binding.E_ALIGN), (dict(ins=12), binding.E_ALIGN), (dict(outs=20), binding.E_ALIGN), (dict(row_stride=20, expert_stride=480), binding.E_ALIGN),
           (dict(expert_stride=24 * 16 + 4), binding.E_ALIGN)]
    for changes, code in bad:
        assert forward(w=_experts(**changes)) == code and back_input(w=_experts(**changes)) == code and back_weights(w=_experts(**changes)) == code
    assert forward(w=_experts(type=binding.F32)) == binding.E_NOT_IMPLEMENTED and back_input(w=_experts(type=binding.F32)) == binding.E_NOT_IMPLEMENTED
    assert forward(x=_matrix(type=binding.F32)) == binding.E_NOT_IMPLEMENTED and back_weights(x=_matrix(type=binding.F32)) == binding.E_NOT_IMPLEMENTED
    assert forward(x=_matrix(data=FAKE + 2)) == binding.E_ALIGN and forward(x=_matrix(row_stride=20)) == binding.E_ALIGN and forward(x=_matrix(cols=12)) == binding.E_ALIGN
    assert forward(x=_matrix(cols=8)) == binding.E_BAD_PARAM and forward(x=_matrix(type=binding.F16)) == binding.E_BAD_PARAM
    assert forward(per_row=0) == binding.E_BAD_PARAM and forward(per_row=1) == binding.E_BAD_PARAM and forward(order=None) == binding.E_BAD_PARAM
    assert forward(order=FAKE + 1) == binding.E_ALIGN and forward(starts=FAKE + 2) == binding.E_ALIGN
    assert forward(y=_matrix(data=far, rows=20, cols=24, row_stride=24, type=binding.F16)) == binding.E_BAD_PARAM
    assert forward(y=_matrix(rows=20, cols=24, row_stride=24)) == binding.E_BAD_PARAM                                 # on x
    assert forward(y=_matrix(data=FAKE + (1 << 24), rows=20, cols=24, row_stride=24)) == binding.E_BAD_PARAM            # on the weights
    assert back_input(gx=_matrix(rows=19)) == binding.E_BAD_PARAM and back_input(gx=_matrix(data=far, rows=20)) == binding.E_BAD_PARAM
    assert back_weights(per_row=3) == binding.E_BAD_PARAM and back_weights(order=None) == binding.E_BAD_PARAM
    assert back_weights(w=_experts(data=far)) == binding.E_BAD_PARAM and back_weights(w=_experts(data=FAKE)) == binding.E_BAD_PARAM
