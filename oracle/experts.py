"""Products of experts, their gradients, rows and moments in 8 bits and the
AdamW step, in 64 bits with numpy: what the operators' tests compare with.

Written from the definitions in include/netsim.h, expert by expert and without
anything the kernels share.  ``*_bound`` next to a result is the sum of the
magnitudes of what was added up for it, which the tests' tolerances need.
"""

from __future__ import annotations

import math

import numpy as np

_erf = np.vectorize(math.erf, otypes=[float])


def activation(kind, g):
    """(act(g), act'(g))."""
    if kind == "silu":
        p = 1 / (1 + np.exp(-g))
        return g * p, p + g * p * (1 - p)
    p = (1 + _erf(g / math.sqrt(2))) / 2
    return g * p, p + g * np.exp(-g * g / 2) / math.sqrt(2 * math.pi)


def segments(offsets, experts, slots):
    """(expert, first slot, end) of every expert with slots."""
    if offsets is None:
        return [(0, 0, slots)] if slots else []
    bounds = np.clip(np.asarray(offsets, dtype=np.int64), 0, slots)
    return [(e, bounds[e], bounds[e + 1]) for e in range(experts) if bounds[e + 1] > bounds[e]]


def by_slot(x, row_of_slot):
    """(the rows of the slots, whether there is one)."""
    if row_of_slot is None:
        return x, np.ones(len(x), bool)
    at = np.asarray(row_of_slot, dtype=np.int64)
    has = (at >= 0) & (at < len(x))
    out = np.zeros((len(at), x.shape[1]))
    out[has] = x[at[has]]
    return out, has


def multiply(x, weights, offsets, row_of_slot, kind=None):
    """Per matrix (x W^T by slot, the same of magnitudes), and gated's or the
    product's result."""
    rows, has = by_slot(x, row_of_slot)
    z = [np.zeros((len(rows), w.shape[1])) for w in weights]
    top = [np.zeros_like(v) for v in z]
    for e, a, b in segments(offsets, len(weights[0]), len(rows)):
        at = np.flatnonzero(has[a:b]) + a
        for w, v, t in zip(weights, z, top):
            v[at] = rows[at] @ w[e].T
            t[at] = np.abs(rows[at]) @ np.abs(w[e]).T
    return z, top, z[0] if kind is None else activation(kind, z[0])[0] * z[1]


def used(offsets, experts, row_of_slot, slots, rows):
    """Whether a slot takes part: it has an expert and a row."""
    out = np.zeros(slots, bool)
    for _, a, b in segments(offsets, experts, slots):
        out[a:b] = True
    if row_of_slot is not None:
        at = np.asarray(row_of_slot)
        out &= (at >= 0) & (at < rows)
    return out


def gradients(x, weights, d, offsets, row_of_slot, slots_of_row):
    """dx and dW from d, one [slots, n] per matrix."""
    rows, has = by_slot(x, row_of_slot)
    dxs = np.zeros((len(rows), x.shape[1]))
    dw = [np.zeros_like(w) for w in weights]
    for e, a, b in segments(offsets, len(weights[0]), len(rows)):
        at = np.flatnonzero(has[a:b]) + a
        for w, g, out in zip(weights, d, dw):
            dxs[at] += g[at] @ w[e]
            out[e] = g[at].T @ rows[at]
    if row_of_slot is None:
        return dxs, dw
    dx = np.zeros_like(x)
    if slots_of_row is not None:
        for r, list_ in enumerate(np.asarray(slots_of_row)):
            for s in list_:
                if 0 <= s < len(dxs):
                    dx[r] += dxs[s]
    return dx, dw


def quantise(x):
    """Rows x [rows, cols] of 32-bit values -> (q, scale), the scale and the
    factor in 32 bits as the definition has them."""
    x = np.asarray(x, dtype=np.float32)
    with np.errstate(invalid="ignore"):
        top = np.maximum(np.abs(x).max(1), np.float32(2.0 ** -100))
    ok = np.isfinite(x).all(1)
    factor = np.where(ok, np.float32(127) / np.where(ok, top, 1), 0).astype(np.float32)
    q = np.zeros(x.shape, dtype=np.int64)
    q[ok] = np.rint((x[ok] * factor[ok, None]).astype(np.float32))
    return q, np.where(ok, top / np.float32(127), np.nan).astype(np.float32)


def product8(q, scale, wq, w_scale, offsets, row_of_slot):
    rows, has = by_slot(np.asarray(q, dtype=np.float64), row_of_slot)
    scales, _ = by_slot(np.asarray(scale, dtype=np.float64)[:, None], row_of_slot)
    y = np.zeros((len(rows), wq.shape[1]))
    for e, a, b in segments(offsets, len(wq), len(rows)):
        at = np.flatnonzero(has[a:b]) + a
        y[at] = (rows[at] @ wq[e].astype(np.float64).T) * scales[at] * w_scale[e].astype(np.float64)
    return y


def adamw(p, g, m, v, step, lr, beta1, beta2, eps, weight_decay, grad_scale=1.0):
    """(p, m, v) after the step."""
    g = g * grad_scale
    m = beta1 * m + (1 - beta1) * g
    v = beta2 * v + (1 - beta2) * g * g
    hat = (m / (1 - beta1 ** step)) / (np.sqrt(v / (1 - beta2 ** step)) + eps)
    return p - lr * weight_decay * p - lr * hat, m, v


# 8-bit floats of 4 exponent and 3 mantissa bits, by their code (no infinities)
def _float8(code):
    e, f = code >> 3 & 15, code & 7
    if e == 15 and f == 7:
        return math.nan
    return math.copysign((f / 8 * 2.0 ** -6) if e == 0 else (1 + f / 8) * 2.0 ** (e - 7), -1 if code & 128 else 1)


FLOAT8 = np.array([_float8(c) for c in range(256)])


def narrow(x, block=256):
    """(values in the 8-bit floats' units, scales) of a flat x, unrounded:
    what a code may be half a step away from."""
    pad = np.concatenate([x, np.zeros(-len(x) % block)]).reshape(-1, block)
    top = np.abs(pad).max(1)
    top = np.where(top < 2.0 ** -100, 0, top)
    return (pad * np.where(top > 0, 448 / np.where(top > 0, top, 1), 0)[:, None]).reshape(-1), top / 448
