"""The operators behind a router in plain float64 numpy, from their formulas."""
import numpy as np


def scores(l, sigmoid):
    l = np.where(np.isnan(l), -np.inf, np.asarray(l, np.float64))
    with np.errstate(all="ignore"):
        if sigmoid:
            return np.where(l >= 0, 1 / (1 + np.exp(-l)), np.exp(l) / (1 + np.exp(l)))
        m = l.max(axis=1, keepdims=True)
        e = np.where(l == m, 1.0, np.exp(l - m))
        e = np.where(np.isneginf(l), 0.0, e)
        z = e.sum(axis=1, keepdims=True)
        return e / np.where(z == 0, 1.0, z)


def route(l, k, sigmoid=False, bias=None, groups=1, keep=1, top=1, renorm=True, scale=1.0):
    """idx, val, one row after the other."""
    l = np.where(np.isnan(l), -np.inf, np.asarray(l, np.float64))
    s = scores(l, sigmoid)
    rows, n = l.shape
    idx, val = np.full((rows, k), -1, np.int32), np.zeros((rows, k))
    for r in range(rows):
        gone = np.isneginf(l[r])
        by = l[r] if bias is None else s[r] + bias.astype(np.float64)
        if bias is not None:
            gone = gone | np.isnan(bias) | np.isneginf(bias)
        best = []
        for g in range(groups):
            mine = [e for e in range(g * n // groups, (g + 1) * n // groups) if not gone[e]]
            of = s[r] if bias is None and top == 2 else by
            largest = sorted((of[e] for e in mine), reverse=True)[:top]
            best.append((-(sum(largest) if largest else -np.inf), g))
        stay = {g for _, g in sorted(best)[:keep]}
        order = sorted((-by[e], e) for e in range(n) if not gone[e] and e // (n // groups) in stay)[:k]
        for j, (_, e) in enumerate(order):
            idx[r, j] = e
        c = idx[r][idx[r] >= 0]
        if c.size:
            w = s[r, c]
            if renorm:
                # relative to the largest, so that scores that are all tiny keep a sum
                lg = log_scores(l[r:r + 1], sigmoid)[0, c]
                with np.errstate(all="ignore"):
                    w = np.where(lg == lg.max(), 1.0, np.exp(lg - lg.max()))
                w = w / w.sum()
            val[r, :c.size] = scale * w
    return idx, val


def log_scores(l, sigmoid):
    l = np.where(np.isnan(l), -np.inf, np.asarray(l, np.float64))
    with np.errstate(all="ignore"):
        if sigmoid:
            return np.where(l == np.inf, 0.0, np.minimum(l, 0) - np.log1p(np.exp(-np.abs(l))))
        return l                                    # (up to a constant of the row, which the quotients do not see)


def route_vjp(l, idx, t, sigmoid=False, renorm=True, scale=1.0):
    """Through the scores (their logarithms where they are renormalised), row by row."""
    s, lg = scores(l, sigmoid), log_scores(l, sigmoid)
    rows, n = s.shape
    grad = np.zeros((rows, n))
    for r in range(rows):
        js = [j for j in range(idx.shape[1]) if 0 <= idx[r, j] < n and lg[r, idx[r, j]] > -np.inf]
        if not js:
            continue
        c = idx[r, js]
        g = np.asarray(t, np.float64)[r, js]
        if renorm:
            with np.errstate(all="ignore"):
                w = np.where(lg[r, c] == lg[r, c].max(), 1.0, np.exp(lg[r, c] - lg[r, c].max()))
            w = w / w.sum()
            g = w * (g - (g * w).sum())             # in log s
        else:
            g = g * s[r, c]
        for e, v in zip(c, g):
            if sigmoid:
                grad[r, e] += v * scores(-np.asarray([[l[r, e]]], np.float64), True)[0, 0]
            else:
                grad[r] -= v * s[r]
                grad[r, e] += v
    return scale * grad


def places(idx, n, capacity=0):
    """slot, source, offset, load."""
    flat = idx.reshape(-1)
    lists = [[p for p in range(flat.size) if flat[p] == e] for e in range(n)]
    load = np.array([len(m) for m in lists], np.int32)
    if capacity:
        lists = [m[:capacity] for m in lists]
    offset = np.concatenate(([0], np.cumsum([len(m) for m in lists]))).astype(np.int32)
    slot, source = np.full(flat.size, -1, np.int32), np.full(flat.size, -1, np.int32)
    for e, m in enumerate(lists):
        for i, p in enumerate(m):
            slot[p] = offset[e] + i
            source[offset[e] + i] = p
    return slot.reshape(idx.shape), source, offset, load


def product(x, w, offset, source, k):
    """out per place (NaN behind the last), and the sum of the terms' absolute values."""
    slots = len(x) if source is None else len(source)
    out = np.full((slots, w.shape[1]), np.nan)
    size = np.full_like(out, np.nan)
    for e in range(w.shape[0]):
        for s in range(offset[e], offset[e + 1]):
            row = x[s if source is None else source[s] // k]
            out[s] = w[e] @ row
            size[s] = np.abs(w[e]) @ np.abs(row)
    return out, size


def product_vjp(x, w, offset, source, k, t):
    """dx per place, dw, and the sums of absolute values of both."""
    slots = t.shape[0]
    dx, sx = np.full((slots, w.shape[2]), np.nan), np.full((slots, w.shape[2]), np.nan)
    dw, sw = np.zeros(w.shape), np.zeros(w.shape)
    for e in range(w.shape[0]):
        for s in range(offset[e], offset[e + 1]):
            row = x[s if source is None else source[s] // k]
            dx[s], sx[s] = t[s] @ w[e], np.abs(t[s]) @ np.abs(w[e])
            dw[e] += np.outer(t[s], row)
            sw[e] += np.abs(np.outer(t[s], row))
    return dx, dw, sx, sw


def combine(y, slot, val):
    rows, k = slot.shape
    out, size = np.zeros((rows, y.shape[1])), np.zeros((rows, y.shape[1]))
    for t in range(rows):
        for j in range(k):
            if 0 <= slot[t, j] < y.shape[0]:
                out[t] += val[t, j] * y[slot[t, j]]
                size[t] += np.abs(val[t, j] * y[slot[t, j]])
    return out, size


def combine_vjp(y, slot, val, g):
    dy, dval, size = np.full(y.shape, np.nan), np.zeros(slot.shape), np.zeros(slot.shape)
    for t in range(slot.shape[0]):
        for j in range(slot.shape[1]):
            if 0 <= slot[t, j] < y.shape[0]:
                dy[slot[t, j]] = val[t, j] * g[t]
                dval[t, j] = g[t] @ y[slot[t, j]]
                size[t, j] = np.abs(g[t]) @ np.abs(y[slot[t, j]])
    return dy, dval, size
