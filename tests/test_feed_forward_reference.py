"""The plain forms that the experts' feed-forward is tested against: activations and gradients against differences, 8-bit rows
against rational arithmetic."""
from fractions import Fraction

import numpy as np
import pytest

from tests import feed_forward_reference as ref


@pytest.mark.parametrize("name", ref.ACTS)
def test_slopes_are_differences(name):
    g = np.linspace(-9.0, 9.0, 181) + 0.01
    d = 1e-5
    numeric = (ref.act(name, g + d)[0] - ref.act(name, g - d)[0]) / (2 * d)
    # the third derivative is below 3 and values below 10: d^2 / 2 and 10 * 2^-52 / d
    assert np.abs(ref.act(name, g)[1] - numeric).max() < 0.5e-10 * 3 + 10 * 2.0 ** -52 / d


def test_activations_far_out():
    for name in ref.ACTS:
        v, s = ref.act(name, np.array([-40.0, 40.0, 0.0]))
        assert abs(v[0]) < 1e-15 and abs(s[0]) < 1e-15 and v[1] == 40.0 and abs(s[1] - 1.0) < 1e-15 and v[2] == 0.0


@pytest.mark.parametrize("name", ref.ACTS)
def test_gradients_are_differences(name):
    r = np.random.default_rng(5)
    n, f, h, k = 3, 4, 5, 2
    x, wg, wu = r.normal(size=(4, h)), r.normal(size=(n, f, h)), r.normal(size=(n, f, h))
    offset, source = np.array([0, 3, 3, 6]), np.array([0, 3, 6, 1, 99, 7, -1, -1])       # an expert without places, one place without
    t = r.normal(size=(8, f))

    def value():
        return np.nansum(t * ref.gated(x, wg, wu, offset, source, k, name)[0])

    dx, dwg, dwu = ref.gated_vjp(x, wg, wu, offset, source, k, name, t)
    xs, there = ref.rows_of(x, offset, source, k)
    full = np.zeros_like(x)
    for s in range(6):
        if there[s]:
            full[source[s] // k] += dx[s]
    assert (dx[4] == 0).all() and (dwg[1] == 0).all()
    d = 1e-5
    for a, grad in ((x, full), (wg, dwg), (wu, dwu)):
        for i in np.ndindex(*a.shape):
            was = a[i]
            a[i] = was + d
            up = value()
            a[i] = was - d
            down = value()
            a[i] = was
            # (values below 100, third derivatives below 1000 here)
            assert abs((up - down) / (2 * d) - grad[i]) < 1000 * d * d + 100 * 2.0 ** -50 / d


def test_quantise():
    r = np.random.default_rng(6)
    x = r.normal(size=(40, 9)).astype(np.float32).astype(np.float64)
    x[0] = 0
    x[1] = np.arange(9) * 0.5 - 2
    x[1, 0] = 127.0                                       # q = x: halves
    x[2, 3], x[3, 4] = np.nan, -np.inf
    x[4] = np.round(x[4] * 4) / 4
    q, scale = ref.quantise(x)
    assert scale[0] == 0 and not q[0].any() and np.isnan(scale[2:4]).all() and not q[2:4].any()
    for i in [1] + list(range(4, 40)):
        top = max(Fraction(abs(v)) for v in x[i])
        assert [round(127 * Fraction(v) / top) for v in x[i]] == q[i].tolist()        # (ties to even)
        assert abs(Fraction(float(scale[i])) - top / 127) <= top / 127 * Fraction(1, 2 ** 24)
