"""The operators on rows chosen by an id, from their definitions in 64 bits (numpy), and how far 32-bit arithmetic may be off."""
import numpy as np

U = 2.0 ** -24                         # half a step of fp32
HALF = {"fp32": U, "bf16": 2.0 ** -9, "fp16": 2.0 ** -12}      # half a step of a type, relative to the next power of two above; 2 x that to the value
TINY = {"fp32": 2.0 ** -150, "bf16": 2.0 ** -134, "fp16": 2.0 ** -25}      # half the smallest step


def rounding(value, dtype):
    return 2.0 * HALF[dtype] * np.abs(value) + TINY[dtype]


def order_ids(ids, span):
    """order (of the ids that are not left out), starts, distinct"""
    ids = np.asarray(ids).reshape(-1)
    there = np.flatnonzero((ids >= 0) & (ids < span))
    order = there[np.argsort(ids[there], kind="stable")]
    starts = np.searchsorted(ids[order], np.arange(span + 1))
    return order, starts, np.unique(ids[there])


def embedding(table, ids, scale):
    there = (ids >= 0) & (ids < table.shape[0])
    out = np.zeros((len(ids), table.shape[1]))
    out[there] = scale * table[ids[there]]
    return out


def embedding_backward(grad, ids, span, scale):
    """The table's gradient, and the sums of magnitudes and the numbers of terms that bound its error."""
    there = (ids >= 0) & (ids < span)
    out, size, terms = np.zeros((span, grad.shape[1])), np.zeros((span, grad.shape[1])), np.zeros(span)
    np.add.at(out, ids[there], grad[there])
    np.add.at(size, ids[there], np.abs(grad[there]))
    np.add.at(terms, ids[there], 1)
    return scale * out, abs(scale) * size, terms


def sum_error(size, terms):
    """fp32 sums of so many terms in any order, times a scale: each addition half a step of at most the sum of magnitudes; one product."""
    return (np.asarray(terms)[:, None] + 2.0) * U * size


def products(x, source, starts, w):
    """forward: y, and the sums of magnitudes"""
    y, size = np.zeros((len(source), w.shape[1])), np.zeros((len(source), w.shape[1]))
    for e in range(w.shape[0]):
        part = slice(starts[e], starts[e + 1])
        y[part] = x[source[part]] @ w[e].T
        size[part] = np.abs(x[source[part]]) @ np.abs(w[e]).T
    return y, size


def products_input(gy, starts, w):
    gx, size = np.zeros((gy.shape[0], w.shape[2])), np.zeros((gy.shape[0], w.shape[2]))
    for e in range(w.shape[0]):
        part = slice(starts[e], starts[e + 1])
        gx[part] = gy[part] @ w[e]
        size[part] = np.abs(gy[part]) @ np.abs(w[e])
    return gx, size


def products_weights(gy, x, source, starts):
    experts = len(starts) - 1
    gw, size = np.zeros((experts, gy.shape[1], x.shape[1])), np.zeros((experts, gy.shape[1], x.shape[1]))
    for e in range(experts):
        part = slice(starts[e], starts[e + 1])
        gw[e] = gy[part].T @ x[source[part]]
        size[e] = np.abs(gy[part]).T @ np.abs(x[source[part]])
    return gw, size


def product_error(size, terms):
    """Products of 16-bit values are exact in fp32.  The tensor cores add 16 of them to the accumulator at a time; each of the 17 terms may be cut
    off at the last bit of the largest, of at most the sum of magnitudes, and so may the result: 18 steps of 2^-23 every 16 terms."""
    return (np.ceil(np.asarray(terms, dtype=np.float64) / 16.0) + 1.0) * 18.0 * 2.0 ** -23 * size
