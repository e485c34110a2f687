"""Operators of an expert-parallel layer in 64 bits on the CPU (numpy),
straight from their definitions and row by row where that is plainest.
"""

from __future__ import annotations

import numpy as np

INF = np.inf
BLOCK = 32


def scores(kind, x):
    """Scores of rows x (float64); 0 where the logit is minus infinity."""
    if kind == "sigmoid":
        with np.errstate(over="ignore"):
            return 1.0 / (1.0 + np.exp(-x))
    top = x.max(1, keepdims=True)
    with np.errstate(invalid="ignore"):
        p = np.where(x == -INF, 0.0, np.exp(x - top))
        z = p.sum(1, keepdims=True)
        return np.where(z == 0, 0.0, p / np.where(z == 0, 1.0, z))


def choice_values(r, x, bias):
    """What the choice compares (-inf: cannot be chosen)."""
    c = x.copy() if bias is None and not (r.groups > 1 and r.group_best > 1) else scores(r.scores, x)
    if bias is not None:
        c = c + bias
    return np.where(x == -INF, -INF, c)


def group_values(r, c):
    """Value of every group of a row of choice values."""
    out = []
    for g in range(r.groups):
        best = sorted(c[g * (r.experts // r.groups):(g + 1) * (r.experts // r.groups)], reverse=True)
        out.append(sum(v for j, v in enumerate(best[:r.group_best]) if j == 0 or v > -INF))
    return out


def route(r, logits, bias=None):
    """(experts, weights) of rows of logits."""
    x = np.asarray(logits, np.float64)
    n = len(x)
    experts, weights = np.full((n, r.top_k), -1), np.zeros((n, r.top_k))
    if not n:
        return experts, weights
    bad = np.isnan(x).any(1) | ((x == INF).any(1) if r.scores == "softmax" else False)
    safe = np.where(bad[:, None], 0.0, x)
    s, c = scores(r.scores, safe), choice_values(r, safe, bias)
    for t in range(n):
        if bad[t]:
            weights[t] = np.nan
            continue
        row = list(c[t])
        if r.groups > 1:
            of = group_values(r, row)
            kept = sorted(range(r.groups), key=lambda g: (-of[g], g))[:r.groups_kept]
            row = [v if e // (r.experts // r.groups) in kept else -INF for e, v in enumerate(row)]
        best = [e for e in sorted(range(r.experts), key=lambda e: (-row[e], e)) if row[e] > -INF][:r.top_k]
        experts[t, :len(best)] = best
        w = s[t, best]
        if r.renormalise and len(best):
            if r.scores == "softmax":     # the scores' ratios, also where they underflow
                w = np.exp(safe[t, best] - safe[t, best].max())
            w = w / w.sum() if w.sum() > 0 else w * 0
        weights[t, :len(best)] = w * r.scale
    return experts, weights


def weights_of(r, x, experts):
    """Weights of a given choice, differentiable formula in 64 bits (one row)."""
    s = scores(r.scores, x[None])[0][experts]
    return r.scale * (s / s.sum() if r.renormalise else s)


def route_backward(r, logits, experts, dweights):
    x = np.asarray(logits, np.float64)
    out = np.zeros_like(x)
    s = scores(r.scores, x)
    for t in range(len(x)):
        j = np.flatnonzero(experts[t] >= 0)
        e, dw = experts[t][j], r.scale * np.asarray(dweights, np.float64)[t][j]
        if not len(e):
            continue
        p = s[t, e]
        if r.renormalise:
            z = p.sum()
            if z == 0:          # the weights are 0 whatever the logits
                continue
            dp = (dw - (dw * p).sum() / z) / z
        else:
            dp = dw
        if r.scores == "sigmoid":
            with np.errstate(over="ignore"):
                out[t, e] = dp * p / (1 + np.exp(x[t, e]))
        else:
            out[t] = -s[t] * (dp * p).sum()
            out[t, e] += dp * p
    return out


def dispatch(experts, num_experts, ranks, per_rank, row_bytes, once):
    tokens, k = experts.shape
    slots = [[] for _ in range(num_experts)]
    sent = np.zeros((ranks, ranks))
    for t in range(tokens):
        seen = set()
        for j in range(k):
            e = int(experts[t, j])
            if not 0 <= e < num_experts:
                continue
            slots[e].append((t, j))
            to = e // (num_experts // ranks)
            if not (once and to in seen):
                sent[t // per_rank, to] += 1
            seen.add(to)
    offsets = np.concatenate([[0], np.cumsum([len(s) for s in slots])])
    order = [x for s in slots for x in s]
    token, slot = np.full(tokens * k, -1), np.full((tokens, k), -1)
    for i, (t, j) in enumerate(order):
        token[i], slot[t, j] = t, i
    return offsets, token, slot, sent * row_bytes


def save(x):
    """(q, exponents) of rows x; exponents of blocks of zeros are -126."""
    x = np.asarray(x, np.float64)
    rows, cols = x.shape
    blocks = -(-cols // BLOCK)
    pad = np.zeros((rows, blocks * BLOCK))
    pad[:, :cols] = x
    pad = pad.reshape(rows, blocks, BLOCK)
    odd = ~np.isfinite(pad).all(2)
    pad = np.where(odd[:, :, None], 0.0, pad)
    e = np.maximum(np.frexp(np.abs(pad).max(2))[1] - 1 - 6, -126)
    e = np.where((pad == 0).all(2), -126, e)
    q = np.clip(np.rint(pad * np.exp2(-e.astype(np.float64))[:, :, None]), -127, 127)
    return q.reshape(rows, blocks * BLOCK).astype(np.int8), np.where(odd, -128, e).astype(np.int8)


def restore(q, e, cols):
    step = np.where(e == -128, np.nan, np.exp2(e.astype(np.float64)))
    return (q.astype(np.float64).reshape(*e.shape, BLOCK) * step[:, :, None]).reshape(q.shape)[:, :cols]


def weight_grad(x, dy, offsets, rows):
    """x: restored rows; rows: row of every slot (out of range: zeros)."""
    x, dy = np.asarray(x, np.float64), np.asarray(dy, np.float64)
    out = np.zeros((len(offsets) - 1, dy.shape[1], x.shape[1]))
    for e in range(len(out)):
        s = np.arange(offsets[e], offsets[e + 1])
        s = s[(rows[s] >= 0) & (rows[s] < len(x))]
        out[e] = dy[s].T @ x[rows[s]]
    return out
