"""The experts' feed-forward in plain float64 numpy, from its formulas."""
import numpy as np
from scipy.special import erfc, expit

ACTS = ("silu", "gelu", "gelu_tanh", "relu")
C = np.sqrt(2.0 / np.pi)


def act(name, g):
    """Value and derivative."""
    g = np.asarray(g, np.float64)
    if name == "relu":
        return np.where(g <= 0, 0.0, g), np.where(g <= 0, 0.0, 1.0)
    if name == "gelu":
        p, d = 0.5 * erfc(-g / np.sqrt(2.0)), np.exp(-0.5 * g * g) / np.sqrt(2.0 * np.pi)
        return g * p, p + g * d
    z, dz = (g, 1.0) if name == "silu" else (2.0 * C * (g + 0.044715 * g ** 3), 2.0 * C * (1.0 + 3 * 0.044715 * g * g))
    p = expit(z)
    return g * p, p + g * p * expit(-z) * dz


def rows_of(x, offset, source, k):
    """The row of x behind every place, zeros where its source is out of range."""
    if source is None:
        return x, np.ones(len(x), bool)
    row = np.asarray(source, np.int64) // k
    there = (np.asarray(source) >= 0) & (row < len(x))
    out = np.zeros((len(source), x.shape[1]))
    out[there] = x[row[there]]
    return out, there


def sums(xs, w, offset):
    """W[e] x per place (NaN behind the last), and the sums of absolute values."""
    out = np.full((len(xs), w.shape[1]), np.nan)
    size = np.full_like(out, np.nan)
    for e in range(w.shape[0]):
        part = slice(offset[e], offset[e + 1])
        out[part] = xs[part] @ w[e].T
        size[part] = np.abs(xs[part]) @ np.abs(w[e]).T
    return out, size


def gated(x, wg, wu, offset, source, k, name):
    xs, _ = rows_of(x, offset, source, k)
    g, u = sums(xs, wg, offset)[0], sums(xs, wu, offset)[0]
    return act(name, g)[0] * u, g, u


def back(dg, du, xs, wg, wu, offset):
    """dx per place, dWg, dWu of given slopes."""
    dx = np.full((len(xs), wg.shape[2]), np.nan)
    dwg, dwu = np.zeros(wg.shape), np.zeros(wu.shape)
    for e in range(wg.shape[0]):
        part = slice(offset[e], offset[e + 1])
        dx[part] = dg[part] @ wg[e] + du[part] @ wu[e]
        dwg[e], dwu[e] = dg[part].T @ xs[part], du[part].T @ xs[part]
    return dx, dwg, dwu


def gated_vjp(x, wg, wu, offset, source, k, name, t, pre=None):
    """dx per place, dWg, dWu, from the sums or from given ones; rows whose source is out of range add nothing."""
    xs, there = rows_of(x, offset, source, k)
    _, g, u = gated(x, wg, wu, offset, source, k, name)
    if pre is not None:
        g, u = pre[:, 0], pre[:, 1]
    value, slope = act(name, g)
    with np.errstate(invalid="ignore"):
        dg, du = np.where(there[:, None], t * u * slope, 0.0), np.where(there[:, None], t * value, 0.0)
    return back(dg, du, xs, wg, wu, offset)


def quantise(x):
    """q, scale of values that float32 holds; the exact quotient's nearest integer, ties to even."""
    a = np.abs(x).max(axis=1)
    ok = np.isfinite(a)
    q = np.zeros(x.shape, np.int8)
    some = ok & (a > 0)
    q[some] = np.rint(127.0 * x[some] / a[some, None])
    with np.errstate(invalid="ignore"):
        return q, np.where(ok, np.float32(a) / np.float32(127.0), np.float32("nan"))
