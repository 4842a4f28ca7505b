"""The losses on logits in 64 bits, from their definitions, on the CPU (numpy), and how far 32-bit arithmetic may be off.

Nothing here is shared with the library or with the measured plain forms."""
from __future__ import annotations

import numpy as np

U = 2.0 ** -24                    # half a step of fp32, relative
EX2 = 2.0 ** -22                  # relative error of the hardware's 2^x (two ulp), which the kernels use
HALF_STEP = {"fp32": 2.0 ** -24, "bf16": 2.0 ** -8, "fp16": 2.0 ** -11}
LEAST = {"fp32": 2.0 ** -149, "bf16": 2.0 ** -133, "fp16": 2.0 ** -24}      # the types' smallest steps


def top(z, k, temperature=1.0):
    """keys, values, lse, tail of z [rows, cols] (float64 that holds the exact values)."""
    rows, cols = z.shape
    keys = np.empty((rows, k), np.int64)
    lse, tail = np.empty(rows), np.empty(rows)
    for r in range(rows):
        x = z[r] + 0.0                                      # -0 -> 0
        order = np.lexsort((np.arange(cols), -np.where(np.isnan(x), 0.0, x), ~np.isnan(x)))     # NaN first, then descending, then by column
        keys[r] = order[:k]
        lse[r], tail[r] = _lse(x / temperature), 0.0
        if np.isnan(lse[r]) or lse[r] == np.inf:
            lse[r] = tail[r] = np.nan
        elif lse[r] > -np.inf and k < cols:
            tail[r] = np.exp(_lse(x[order[k:]] / temperature) - lse[r])
    return keys, np.take_along_axis(z, keys, 1), lse, tail


def _lse(x):
    if np.isnan(x).any():
        return np.nan
    m = x.max() if x.size else -np.inf
    return m if np.isinf(m) else m + np.log(np.exp(x - m).sum())


def distill(z, keys, values, temperature=1.0, tail=None, weight=None):
    """(loss [rows], gradient [rows, cols], scale of the gradient's 32-bit error [rows, cols], of the loss's [rows])."""
    rows, cols = z.shape
    t = float(temperature)
    loss, grad = np.zeros(rows), np.zeros((rows, cols))
    grad_err, loss_err = np.zeros((rows, cols)), np.zeros(rows)
    for r in range(rows):
        w = 1.0 if weight is None else float(weight[r])
        here = (keys[r] >= 0) & (keys[r] < cols)
        if w == 0.0 or not here.any() or np.all(values[r][here] == -np.inf) or np.all(z[r] == -np.inf):
            continue
        a = 0.0 if tail is None else float(tail[r])
        # (relative to the largest: the logarithm of a sum would drown in a logit of 10^38)
        key, y, yt = keys[r][here].astype(np.int64), (z[r] - z[r].max()) / t, values[r][here] / t
        with np.errstate(divide="ignore", invalid="ignore"):
            log_p = yt - _lse(yt) + np.log1p(-a)
            log_q = y - _lse(y)
            p = np.exp(log_p)
            terms = np.where(p == 0, 0.0, p * (log_p - log_q[key]))
            target = np.zeros(cols)
            np.add.at(target, key, p)
            g = np.exp(log_q) - target
            total = terms.sum()
            others = np.ones(cols, bool)
            others[key] = False
            r_j = np.zeros(cols)
            if a != 0.0:
                log_rest = _lse(log_q[others]) if others.any() else -np.inf
                total += a * (np.log(a) - log_rest)
                if log_rest > -np.inf:
                    r_j = np.where(others, np.exp(log_q - log_rest), 0.0)
                    g = g - a * r_j
        loss[r], grad[r] = w * t * t * total, w * t * g
        # An exponential of a difference d (in units of the temperature): 2^x is off by EX2; its argument by three roundings of d log2 e (the
        # difference, 1 / T in the factor, the product), which is 3 U |d| of the result.  A sum of n of them, in 512 threads of
        # several partial sums and a tree of at most 16 levels, adds (n / 512 + 24) U; a quotient, a product and a logarithm 8 U.
        finite = y[np.isfinite(y)]
        ft = yt[np.isfinite(yt)]
        d = np.minimum(finite.max() - finite, 104.0).max() if finite.size else 0.0      # (what lies further down is below 2^-149 of the sum)
        dt = np.minimum(ft.max() - ft, 104.0).max() if ft.size else 0.0
        unit = 2.0 * EX2 + (6.0 * (d + dt) + cols / 512.0 + len(key) + 40.0) * U          # of a probability, relative
        grad_err[r] = abs(w) * t * unit * (np.exp(log_q) + target + a * r_j + (a + np.exp(log_q).sum()) * r_j)
        logs = np.abs(np.where(p > 0, log_p - log_q[key], 0.0))
        logs = logs[np.isfinite(logs)]
        loss_err[r] = abs(w) * t * t * ((1.0 + (logs.max() if logs.size else 0.0)) * unit + 8.0 * U * (d + dt + np.log(cols) + 4.0))
    return loss, grad, grad_err, loss_err


def counts(selected, experts, mask=None, offsets=None):
    tokens = selected.shape[0]
    offsets = [0, tokens] if offsets is None else [int(o) for o in offsets]
    keep = np.ones(tokens, bool) if mask is None else mask.astype(bool)
    out, counted = np.zeros((len(offsets) - 1, experts), np.int64), np.zeros(len(offsets) - 1, np.int64)
    for s, (a, b) in enumerate(zip(offsets[:-1], offsets[1:])):
        for t in range(a, b):
            if keep[t]:
                counted[s] += 1
                for e in selected[t]:
                    if 0 <= e < experts:
                        out[s, e] += 1
    return out, counted


def balance(x, count, counted, coef=1.0, mask=None, offsets=None, grad_loss=None):
    """(loss [segments], gradient, scale of the gradient's error, of the loss's); NaN in the gradient's rows of tokens without a segment."""
    tokens, experts = x.shape
    offsets = [0, tokens] if offsets is None else [int(o) for o in offsets]
    keep = np.ones(tokens, bool) if mask is None else mask.astype(bool)
    loss, grad = np.zeros(len(offsets) - 1), np.full((tokens, experts), np.nan)
    grad_err, loss_err = np.zeros((tokens, experts)), np.zeros(len(offsets) - 1)
    for s, (a, b) in enumerate(zip(offsets[:-1], offsets[1:])):
        f = count[s] / count[s].sum() if count[s].sum() else np.zeros(experts)
        scale = coef * experts / counted[s] if counted[s] else 0.0
        up = 1.0 if grad_loss is None else float(grad_loss[s])
        for t in range(a, b):
            grad[t] = 0.0
            if not keep[t] or np.all(x[t] == -np.inf):
                continue
            d = x[t] - x[t].max()
            p = np.exp(d)
            p = p / p.sum()
            dot = (f * p).sum()
            loss[s] += scale * dot
            grad[t] = up * scale * p * (f - dot)
            # as above: an exponential, a sum over at most 1024 experts in 32 lanes, two quotients and four products
            unit = 2.0 * EX2 + (6.0 * np.minimum(-d, 104.0).max() + 2.0 * (experts / 32.0 + 5.0) + 16.0) * U
            grad_err[t] = abs(up * scale) * unit * p * (f + dot)
            loss_err[s] += abs(scale) * unit * dot
    return loss, grad, grad_err, loss_err
