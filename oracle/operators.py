"""64-bit plain implementations (numpy) of the routed and 4-bit operators, for
the tests: written from their definitions, row by row where that is plainer."""
from __future__ import annotations

import math

import numpy as np

E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def scores(logits, score):
    """Scores of one row of logits (float64), -inf scoring 0."""
    if score == "softmax":
        e = np.exp(logits - logits.max())
        return e / e.sum()
    with np.errstate(over="ignore"):
        return 1.0 / (1.0 + np.exp(-logits))


def _largest(keys, n):
    """Indices of the n largest finite-or-inf keys above -inf, descending, ties
    to the lowest index; -1 where there are none left."""
    order = sorted((i for i in range(len(keys)) if keys[i] > -math.inf), key=lambda i: (-keys[i], i))
    return (order + [-1] * n)[:n]


def route_row(logits, k, score="softmax", bias=None, groups=1, top_groups=1, group_top=1, renorm=True, scale=1.0):
    l = np.asarray(logits, np.float64)
    E = len(l)
    b = None if bias is None else np.asarray(bias, np.float64)
    if np.isnan(l).any() or (b is not None and np.isnan(b).any()) or (score == "softmax" and (l == np.inf).any()):
        return np.full(k, np.nan), [-1] * k
    if (l == -np.inf).all():
        return np.zeros(k), [-1] * k
    s = scores(l, score)
    if b is None and (group_top == 1 or groups == 1):
        key = l.copy()
    else:
        key = s + (0 if b is None else b)
        key[l == -np.inf] = -np.inf
    if groups > 1:
        gs = E // groups
        value = []
        for g in range(groups):
            top = [key[g * gs + i] for i in _largest(key[g * gs:(g + 1) * gs], min(group_top, gs)) if i >= 0]
            value.append(sum(top) if top else -math.inf)
        stay = _largest(value, top_groups)
        for g in range(groups):
            if g not in stay:
                key[g * gs:(g + 1) * gs] = -np.inf
    ids = _largest(key, k)
    w = np.array([s[i] if i >= 0 else 0.0 for i in ids])
    if renorm:
        # relative to the largest chosen, so that scores that underflow keep their ratios
        have = [i for i in ids if i >= 0]
        m = max((l[i] for i in have), default=0.0)
        c = min(m, 0.0) if score == "sigmoid" else m
        e = np.array([0.0 if i < 0 else np.exp(l[i] - c) / (1 + np.exp(l[i])) if score == "sigmoid" and c < 0
                      else s[i] if score == "sigmoid" else np.exp(l[i] - c) for i in ids])
        w = e / e.sum() if have else e
    return w * scale, ids


def route(logits, k, **how):
    rows = [route_row(r, k, **how) for r in np.asarray(logits, np.float64)]
    return (np.array([r[0] for r in rows]).reshape(len(rows), k),
            np.array([r[1] for r in rows], np.int32).reshape(len(rows), k))


def route_weights(logits, ids, score="softmax", renorm=True, scale=1.0):
    """The weights alone, the choice given (what the gradient is of)."""
    out = np.zeros(ids.shape)
    for t, (l, row) in enumerate(zip(np.asarray(logits, np.float64), ids)):
        s = scores(l, score)
        w = np.array([s[i] if 0 <= i < len(l) else 0.0 for i in row])
        out[t] = scale * (w / w.sum() if renorm and w.sum() > 0 else w)
    return out


def route_backward(logits, ids, dw, score="softmax", renorm=True, scale=1.0):
    """d(sum w dw) / d logits through the Jacobians of each step."""
    l = np.asarray(logits, np.float64)
    out = np.zeros_like(l)
    for t in range(len(l)):
        s = scores(l[t], score)
        have = [j for j, i in enumerate(ids[t]) if 0 <= i < l.shape[1]]
        if not have:
            continue
        c = s[ids[t][have]]
        g = scale * np.asarray(dw, np.float64)[t][have]
        if renorm:
            g = (g - (g * c).sum() / c.sum()) / c.sum()
        ds = np.zeros(l.shape[1])
        np.add.at(ds, ids[t][have], g)
        out[t] = s * (ds - (s * ds).sum()) if score == "softmax" else s * (1 - s) * ds
    return out


def plan(ids, E):
    """(order, pos, offsets): order holds the filled slots alone."""
    flat = np.asarray(ids).reshape(-1)
    order = np.array([i for e in range(E) for i in np.flatnonzero(flat == e)], np.int32)
    pos = np.full(flat.shape, -1, np.int32)
    pos[order] = np.arange(len(order), dtype=np.int32)
    counts = [(flat == e).sum() for e in range(E)]
    return order, pos.reshape(np.asarray(ids).shape), np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)


def expert_rows(x, w, bias, order, offsets, k, sorted_rows=False, relu=False):
    """(rows, magnitudes): the filled sorted rows, and the sums of the terms' magnitudes."""
    n = int(offsets[-1])
    y, mag = np.zeros((n, w.shape[1])), np.zeros((n, w.shape[1]))
    for e in range(w.shape[0]):
        r = np.arange(offsets[e], offsets[e + 1])
        xe = x[r if sorted_rows else order[r] // k]
        y[r] = xe @ w[e].T + (0 if bias is None else bias[e])
        mag[r] = np.abs(xe) @ np.abs(w[e]).T + (0 if bias is None else np.abs(bias[e]))
    return (np.maximum(y, 0) if relu else y), mag


def expert_grads(dy, x, w, order, offsets, k, sorted_rows=False, relu_input=False):
    """((dx, dw, db), their magnitudes) over the filled sorted rows."""
    n = int(offsets[-1])
    E, N, K = w.shape
    out = [np.zeros((n, K)), np.zeros((E, N, K)), np.zeros((E, N))]
    mag = [np.zeros_like(o) for o in out]
    for e in range(E):
        r = np.arange(offsets[e], offsets[e + 1])
        xe, d = x[r if sorted_rows else order[r] // k], dy[r]
        keep = xe > 0 if relu_input else np.ones_like(xe)
        out[0][r], mag[0][r] = (d @ w[e]) * keep, np.abs(d) @ np.abs(w[e])
        out[1][e], mag[1][e] = d.T @ xe, np.abs(d).T @ np.abs(xe)
        out[2][e], mag[2][e] = d.sum(0), np.abs(d).sum(0)
    return out, mag


def mx4_quantize(x):
    """(values, codes, scales) of rows x [rows][K], in the padded layout."""
    x = np.asarray(x, np.float64)
    rows, K = x.shape
    Kp = (K + 127) // 128 * 128
    v = np.zeros((rows, Kp))
    v[:, :K] = x
    code = np.zeros((rows, Kp), np.uint8)
    scale = np.zeros((rows, Kp // 32), np.uint8)
    values = np.zeros((rows, Kp))
    for r in range(rows):
        for b in range(Kp // 32):
            block = v[r, 32 * b:32 * b + 32]
            if not np.isfinite(block).all():
                scale[r, b] = 255
                values[r, 32 * b:32 * b + 32] = np.nan
                continue
            top = np.abs(block).max()
            X = max(math.frexp(top)[1] - 3, -127) if top > 0 else -127
            scale[r, b] = X + 127
            for i, f in enumerate(block):
                a = abs(f) * 2.0 ** -X
                best = min(range(8), key=lambda q: (abs(a - E2M1[q]), q % 2))
                sign = 8 if math.copysign(1.0, f) < 0 else 0
                code[r, 32 * b + i] = best | sign
                values[r, 32 * b + i] = math.copysign(E2M1[best], f) * 2.0 ** X
    return values[:, :K], code[:, 0::2] | (code[:, 1::2] << 4), scale
