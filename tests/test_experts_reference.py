"""The plain float64 forms of the operators behind a router against worked values and differences, and the refusals of the
entry points that need no GPU."""
import ctypes

import numpy as np
import pytest

from tests import experts_reference as ref
from tests.test_abi import lib  # noqa: F401  (the fixture)


def test_route_worked_values():
    l = np.log(np.array([[4.0, 1.0, 3.0, 2.0]]))
    idx, val = ref.route(l, 2)
    assert idx.tolist() == [[0, 2]] and np.allclose(val, [[4 / 7, 3 / 7]])
    idx, val = ref.route(l, 2, renorm=False, scale=2.0)
    assert np.allclose(val, [[0.8, 0.6]])
    idx, val = ref.route(l, 2, bias=np.array([0.0, 0.5, 0.0, 0.0]))          # 0.1 + 0.5 beats 0.4: the weights stay s
    assert idx.tolist() == [[1, 0]] and np.allclose(val, [[0.2, 0.8]])
    idx, _ = ref.route(l, 2, groups=2, keep=1, top=1)
    assert idx.tolist() == [[0, 1]]
    idx, _ = ref.route(np.log(np.array([[4.0, 0.5, 3.0, 2.5]])), 2, groups=2, keep=1, top=2)     # 4.5 < 5.5
    assert idx.tolist() == [[2, 3]]
    idx, val = ref.route(np.array([[0.0, -np.inf, np.nan, -np.inf]]), 2)
    assert idx.tolist() == [[0, -1]] and val.tolist() == [[1.0, 0.0]]
    idx, val = ref.route(np.full((1, 4), -np.inf), 2)
    assert idx.tolist() == [[-1, -1]] and val.tolist() == [[0.0, 0.0]]
    idx, _ = ref.route(np.array([[1.0, 2.0, 2.0, 2.0]]), 2)                   # ties: the lower index
    assert idx.tolist() == [[1, 2]]
    assert np.allclose(ref.route(np.array([[-1000.0, -1000.0]]), 2, sigmoid=True)[1], 0.5)


@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("renorm", [False, True])
def test_route_vjp_against_differences(sigmoid, renorm):
    r = np.random.default_rng(5)
    l, t = r.normal(size=(3, 7)), r.normal(size=(3, 3))
    idx, _ = ref.route(l, 3, sigmoid, renorm=renorm, scale=1.5)
    idx[1, 2] = -1

    def value(x):
        s = ref.scores(x, sigmoid)
        there = idx >= 0
        w = np.where(there, np.take_along_axis(s, np.where(there, idx, 0), 1), 0.0)
        if renorm:
            w = w / w.sum(axis=1, keepdims=True)
        return 1.5 * (w * t).sum()

    got = ref.route_vjp(l, idx, t, sigmoid, renorm, 1.5)
    for i in np.ndindex(*l.shape):
        d = np.zeros_like(l)
        d[i] = 1e-6
        assert abs((value(l + d) - value(l - d)) / 2e-6 - got[i]) < 1e-8, i


def test_places_worked_values():
    idx = np.array([[2, 0], [2, 5], [0, 2], [-1, 2]], np.int32)
    slot, source, offset, load = ref.places(idx, 3)
    assert offset.tolist() == [0, 2, 2, 6] and load.tolist() == [2, 0, 4]
    assert slot.tolist() == [[2, 0], [3, -1], [1, 4], [-1, 5]] and source.tolist() == [1, 4, 0, 2, 5, 7, -1, -1]
    slot, source, offset, load = ref.places(idx, 3, capacity=2)
    assert offset.tolist() == [0, 2, 2, 4] and load.tolist() == [2, 0, 4]
    assert slot.tolist() == [[2, 0], [3, -1], [1, -1], [-1, -1]] and source.tolist() == [1, 4, 0, 2, -1, -1, -1, -1]


def test_gradients_of_the_sums_against_differences():
    r = np.random.default_rng(6)
    idx = np.array([[0, 2], [2, -1], [1, 0]], np.int32)
    slot, source, offset, _ = ref.places(idx, 3)
    x, w, val = r.normal(size=(3, 4)), r.normal(size=(3, 5, 4)), r.normal(size=(3, 2))
    g = r.normal(size=(3, 5))

    def out(x, w, val):
        y = np.nan_to_num(ref.product(x, w, offset, source, 2)[0])
        return ref.combine(y, slot, val)[0]

    y = np.nan_to_num(ref.product(x, w, offset, source, 2)[0])
    dy, dval, _ = ref.combine_vjp(y, slot, val, g)
    dxs, dw, _, _ = ref.product_vjp(x, w, offset, source, 2, np.nan_to_num(dy))
    dx = ref.combine(np.nan_to_num(dxs), slot, np.ones_like(val))[0]
    for a, d in ((x, dx), (w, dw), (val, dval)):
        for i in np.ndindex(*a.shape):
            keep = a[i]
            a[i] = keep + 1e-6
            hi = (out(x, w, val) * g).sum()
            a[i] = keep - 1e-6
            lo = (out(x, w, val) * g).sum()
            a[i] = keep
            assert abs((hi - lo) / 2e-6 - d[i]) < 1e-7, i


def test_refusals(lib):
    from paper_2302_01425_amd import binding as b
    one = ctypes.c_void_p(256)          # never dereferenced: validation happens first

    def route(type=0, stride=8, rows=4, n=8, k=2, score=0, groups=1, keep=1, top=1, scale=1.0, x=one, idx=one, val=one):
        return lib.topk_route_fwd(x, type, stride, None, rows, n, k, score, groups, keep, top, 1, scale, idx, val, None)
    assert route(rows=0) == 0
    for bad in (dict(type=3), dict(type=-1), dict(stride=-1), dict(rows=-1), dict(rows=1 << 31), dict(n=0), dict(n=1025, k=2),
                dict(k=0), dict(k=9), dict(n=100, k=65), dict(score=2), dict(groups=3), dict(groups=0), dict(groups=2, keep=3),
                dict(groups=2, keep=0), dict(top=3), dict(top=0), dict(groups=4, keep=1, k=3), dict(scale=float("nan")),
                dict(scale=float("inf")), dict(n=130, groups=65)):
        assert route(**bad) == -1, bad
    for bad in (dict(x=None), dict(idx=None), dict(val=None)):
        assert route(**bad) == -2, bad
    v = lib.topk_route_vjp
    assert v(one, 0, 8, one, one, 0, 8, 2, 0, 1, 1.0, one, None) == 0
    assert v(one, 0, 8, one, one, 4, 8, 9, 0, 1, 1.0, one, None) == -1
    assert v(one, 0, 8, one, one, 4, 8, 2, 5, 1, 1.0, one, None) == -1
    for i in (0, 3, 4, 11):
        args = [one, 0, 8, one, one, 4, 8, 2, 0, 1, 1.0, one, None]
        args[i] = None
        assert v(*args) == -2, i

    m = lib.topk_expert_map
    assert lib.topk_expert_map_bytes(64, 2, 64) == 0 and lib.topk_expert_map_bytes(1 << 20, 2, 64) > 0
    assert lib.topk_expert_map_bytes(1 << 30, 2, 64) == 0 and lib.topk_expert_map_bytes(4, 2, 2000) == 0
    assert m(one, -1, 2, 8, 0, one, one, one, one, None, 0, None) == -1
    assert m(one, 4, 0, 8, 0, one, one, one, one, None, 0, None) == -1
    assert m(one, 4, 2, 0, 0, one, one, one, one, None, 0, None) == -1
    assert m(one, 4, 2, 1025, 0, one, one, one, one, None, 0, None) == -1
    assert m(one, 1 << 30, 2, 8, 0, one, one, one, one, None, 0, None) == -1
    assert m(one, 4, 2, 8, -1, one, one, one, one, None, 0, None) == -1
    assert m(one, 4, 2, 8, 0, one, one, None, one, None, 0, None) == -2
    assert m(None, 4, 2, 8, 0, one, one, one, one, None, 0, None) == -2
    assert m(one, 1 << 20, 2, 8, 0, one, one, one, one, None, 0, None) == -4
    assert m(one, 1 << 20, 2, 8, 0, one, one, one, one, one, 16, None) == -4

    def product(stride=8, rows=4, we=64, wo=8, wi=1, offset=one, source=one, k=2, slots=8, n=3, h=8, ho=8, type=0, x=one, w=one,
                out=one):
        return lib.topk_expert_product_fwd(x, stride, rows, w, we, wo, wi, offset, source, k, slots, n, h, ho, type, out, None)
    assert product(slots=0) == 0
    for bad in (dict(stride=-1), dict(rows=-1), dict(wo=2, wi=2), dict(we=-1), dict(k=0), dict(slots=-1), dict(slots=1 << 31),
                dict(n=0), dict(n=1025), dict(h=0), dict(ho=0), dict(type=7), dict(source=None, rows=7)):
        assert product(**bad) == -1, bad
    for bad in (dict(offset=None), dict(x=None), dict(w=None), dict(out=None)):
        assert product(**bad) == -2, bad

    def product_vjp(t=one, ts=8, dx=one, dw=one, x=one, w=one):
        return lib.topk_expert_product_vjp(x, 8, 4, w, 64, 8, 1, one, one, 2, 8, 3, 8, 8, 0, t, ts, dx, dw, None)
    assert product_vjp(ts=-1) == -1
    assert product_vjp(t=None) == -2 and product_vjp(dx=None, dw=None) == -2 and product_vjp(x=None) == -2
    assert product_vjp(w=None) == -2

    c = lib.topk_combine_fwd
    assert c(one, 8, one, one, 0, 2, 8, 8, 0, one, None) == 0
    for args in ((8, 4, 0, 8, 8, 0), (8, -1, 2, 8, 8, 0), (8, 4, 2, -1, 8, 0), (8, 4, 2, 8, 0, 0), (-1, 4, 2, 8, 8, 0),
                 (8, 4, 2, 8, 8, 9)):
        assert c(one, args[0], one, one, *args[1:], one, None) == -1, args
    assert c(None, 8, one, one, 4, 2, 8, 8, 0, one, None) == -2
    assert c(one, 8, None, one, 4, 2, 8, 8, 0, one, None) == -2
    assert c(one, 8, one, one, 4, 2, 8, 8, 0, None, None) == -2
    cv = lib.topk_combine_vjp
    assert cv(one, 8, one, one, one, 8, 4, 2, 8, 8, 0, one, None, None) == -2         # weights without their gradient
    assert cv(one, 8, one, one, None, 8, 4, 2, 8, 8, 0, one, one, None) == -2
    assert cv(one, 8, one, one, one, 8, 4, 2, 8, 8, 0, None, one, None) == -2
    assert cv(one, 8, one, one, one, -8, 4, 2, 8, 8, 0, one, one, None) == -1


def test_binding_refuses_cpu_tensors(lib):
    import torch
    from paper_2302_01425_amd import binding as b
    f, i = torch.zeros(4, 8), torch.zeros(4, 2, dtype=torch.int32)
    for call in (lambda: b.topk_route_fwd(f, 2), lambda: b.topk_route_vjp(f, i, f[:, :2]), lambda: b.topk_expert_map(i, 8),
                 lambda: b.topk_expert_product_fwd(f, torch.zeros(2, 3, 8), torch.zeros(3, dtype=torch.int32)),
                 lambda: b.topk_combine_fwd(f, i), lambda: b.topk_combine_vjp(f, i, None, f)):
        with pytest.raises(b.TopkError):
            call()
