"""Routing of tokens to experts and the tokens' way through the expert buffers (the steps around the expert layers of Sec. 7.6).

    s = softmax(x) | sigmoid(x);  c = s + bias;  groups ranked by the sum of their best one or two c;  the top_k best c of the groups that
    stay, descending, equals by the lower index;  weight = scale * s, divided by the sum over the chosen where asked

An expert whose logit or bias is -inf is never chosen; a choice that finds none is -1 with weight 0.  Without a bias the logits' order is the
scores' order, also inside groups that rank by sums of scores.  Everything is computed token by token, in float64.

    plan      choice n = t * k + i takes the row of its expert's buffer that counts the choices before it; -1 beyond the capacity
    dispatch  X_e[position] = x[t];   combine  out[t] = sum_i w_i Y_e[position]
"""
from __future__ import annotations

import math

import numpy as np


def _scores(x, sigmoid):
    if sigmoid:
        return np.array([1.0 / (1.0 + math.exp(-v)) if v >= 0 else math.exp(v) / (1.0 + math.exp(v)) if v > -700 else 0.0 for v in x])
    m = max(x)
    if m == -math.inf:
        return np.zeros(len(x))
    e = np.exp(np.asarray(x) - m)
    return e / e.sum()


def choose(x, top_k, sigmoid=False, bias=None, groups=1, top_groups=None, group_best=1):
    """The chosen experts of one token, -1 where there is none."""
    E = len(x)
    top_groups = groups if top_groups is None else top_groups
    open_ = [x[e] > -math.inf and (bias is None or bias[e] > -math.inf) for e in range(E)]
    if bias is None and (groups == 1 or group_best == 1):
        c = [float(v) for v in x]
    else:
        s = _scores(x, sigmoid)
        c = [float(s[e]) + (float(bias[e]) if bias is not None else 0.0) for e in range(E)]
    if groups > 1:
        per = E // groups
        score = []
        for g in range(groups):
            members = sorted((c[e] for e in range(g * per, (g + 1) * per) if open_[e]), reverse=True)
            score.append(sum(members[:group_best]) if members else None)
        ranked = sorted((g for g in range(groups) if score[g] is not None), key=lambda g: (-score[g], g))[:top_groups]
        open_ = [open_[e] and e // per in ranked for e in range(E)]
    if bias is None:
        c = [float(v) for v in x]                 # (what the groups' sums were taken of ranks groups only)
    order = sorted((e for e in range(E) if open_[e]), key=lambda e: (-c[e], e))[:top_k]
    return order + [-1] * (top_k - len(order))


def weigh(x, chosen, sigmoid=False, renormalise=False, scale=1.0):
    """Weights of one token's choices."""
    live = [e for e in chosen if e >= 0]
    if not live:
        return np.zeros(len(chosen))
    if renormalise:
        # ratios, with the largest score as the unit (log of a sigmoid: x - log(1 + e^x))
        log = lambda v: (-math.log1p(math.exp(-v)) if v >= 0 else v - math.log1p(math.exp(v))) if sigmoid else v
        top = max(log(x[e]) for e in live)
        r = {e: math.exp(log(x[e]) - top) for e in live}
        total = sum(r[e] for e in live)
        return np.array([scale * r[e] / total if e >= 0 else 0.0 for e in chosen])
    s = _scores(x, sigmoid)
    return np.array([scale * s[e] if e >= 0 else 0.0 for e in chosen])


def route_fwd(logits, top_k, sigmoid=False, bias=None, groups=1, top_groups=None, group_best=1, renormalise=False, scale=1.0):
    """(indices [T x k], weights [T x k])."""
    X = np.asarray(logits, dtype=np.float64)
    idx = np.full((X.shape[0], top_k), -1, dtype=np.int64)
    w = np.zeros((X.shape[0], top_k))
    for t, x in enumerate(X):
        idx[t] = choose(x, top_k, sigmoid, bias, groups, top_groups, group_best)
        w[t] = weigh(x, idx[t], sigmoid, renormalise, scale)
    return idx, w


def route_bwd(logits, indices, dweights, sigmoid=False, renormalise=False, scale=1.0):
    """dlogits, and per logit the sum of the magnitudes of the terms it is made of (what its rounding errors are relative to)."""
    X = np.asarray(logits, dtype=np.float64)
    dX, size = np.zeros_like(X), np.zeros_like(X)
    for t, x in enumerate(X):
        live = [(int(e), float(g)) for e, g in zip(indices[t], dweights[t]) if 0 <= e < X.shape[1] and x[e] > -math.inf]
        if not live:
            continue
        s = _scores(x, sigmoid)
        rest = _scores([-v for v in x], True) if sigmoid else None        # 1 - s, which is below 1's last bit where s is near 1
        if renormalise:
            u = weigh(x, [e for e, _ in live], sigmoid, True, 1.0)
            mean = sum(a * g for a, (_, g) in zip(u, live))
            spread = sum(abs(a * g) for a, (_, g) in zip(u, live))
            for a, (e, g) in zip(u, live):
                f = scale * a * (rest[e] if sigmoid else 1.0)
                dX[t, e] += f * (g - mean)
                size[t, e] += abs(f) * (abs(g) + spread)
        elif sigmoid:
            for e, g in live:
                f = scale * s[e] * rest[e]
                dX[t, e] += f * g
                size[t, e] += abs(f * g)
        else:
            dot = sum(s[e] * g * scale for e, g in live)
            spread = sum(abs(s[e] * g * scale) for e, g in live)
            dX[t] -= s * dot
            size[t] += s * spread
            for e, g in live:
                dX[t, e] += s[e] * g * scale
                size[t, e] += abs(s[e] * g * scale)
    return dX, size


def plan(indices, experts, capacity):
    """(position like indices, rows [E], counts [E])."""
    idx = np.asarray(indices)
    pos = np.full(idx.shape, -1, dtype=np.int64)
    counts = np.zeros(experts, dtype=np.int64)
    for t in range(idx.shape[0]):
        for i in range(idx.shape[1]):
            e = int(idx[t, i])
            if 0 <= e < experts:
                if counts[e] < capacity:
                    pos[t, i] = counts[e]
                counts[e] += 1
    return pos, np.minimum(counts, capacity), counts


def _slots(indices, position, lo, hi, capacity):
    for t in range(indices.shape[0]):
        for i in range(indices.shape[1]):
            e, p = int(indices[t, i]), int(position[t, i])
            if lo <= e < hi and 0 <= p < capacity:
                yield t, i, e, p


def dispatch_fwd(x, indices, position, lo, hi, X):
    """Writes the tokens of the experts [lo, hi) into X [experts x capacity x features] (whole-layer indexing), in place."""
    for t, _, e, p in _slots(indices, position, lo, hi, X.shape[1]):
        X[e, p] = x[t]


def dispatch_bwd(dX, indices, position, lo, hi):
    """The device's part of dx."""
    dx = np.zeros((indices.shape[0], dX.shape[2]))
    for t, _, e, p in _slots(indices, position, lo, hi, dX.shape[1]):
        dx[t] += dX[e, p]
    return dx


def combine_fwd(Y, indices, position, weights, lo, hi):
    """The device's part of out."""
    out = np.zeros((indices.shape[0], Y.shape[2]))
    for t, i, e, p in _slots(indices, position, lo, hi, Y.shape[1]):
        out[t] += weights[t, i] * Y[e, p]
    return out


def combine_bwd(Y, indices, position, weights, dout, lo, hi, dY):
    """Writes dY in place where a choice has a row; returns dweights."""
    dw = np.zeros(indices.shape)
    for t, i, e, p in _slots(indices, position, lo, hi, Y.shape[1]):
        dY[e, p] = weights[t, i] * dout[t]
        dw[t, i] = float(np.dot(dout[t], Y[e, p]))
    return dw
