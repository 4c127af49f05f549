"""The operators behind a router (route, expert map, experts' products, combine) on the GPU against their plain float64
forms (experts_reference.py), each by itself, together, captured, on other streams, and what they refuse.

Tolerances count roundings.  u = 2^-24 is half a step of float32, HALF[type] half a step of the output's type.
  route: exp(l - m) has the rounding of l - m (|l - m| u) and its own (2 u); a sum of n <= 1024 terms is 32 sequential and 6
  tree additions (38 u) of terms whose own errors weigh in by their share (ln 1024 < 7 for the |l - m| part); quotient, scale
  and store 4 u: (D + 56) u with D the largest |l - m| among the chosen.
  products: float32 sums of K terms, every addition off by a step at most: (K + 2) 2u sum|a b|, and the output's rounding.
  combine: k terms, k + 1 roundings each, and the output's."""
import numpy as np
import pytest

from tests import experts_reference as ref

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
HALF = {"float32": 2.0 ** -24, "bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}
TINY = {"float32": 2.0 ** -149, "bfloat16": 2.0 ** -133, "float16": 2.0 ** -25}       # half a step of the smallest numbers
MARK = 77.0


@pytest.fixture(scope="module")
def gpu():
    import torch
    from paper_2302_01425_amd import binding
    assert torch.cuda.is_available()
    binding.load()
    return binding


def put(a, dtype="float32"):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a)).cuda().to(getattr(torch, dtype))


def host(t):
    import torch
    torch.cuda.synchronize()
    return t.detach().cpu().double().numpy() if t.is_floating_point() else t.cpu().numpy()


def rounded(a, dtype):
    """The values of `a` in the type, as float64."""
    return host(put(np.asarray(a, np.float64), dtype))


def within(got, want, bound, what):
    bad = ~(np.abs(got - want) <= bound)
    assert not bad.any(), (what, np.argwhere(bad)[:4].tolist(), got[bad][:4], want[bad][:4], np.broadcast_to(bound, got.shape)[bad][:4])


def strided(a, dtype, pad, shift):
    """`a` as rows `pad` elements apart that start `shift` elements into a buffer of marks."""
    import torch
    rows, n = a.shape
    buf = torch.full((rows * (n + pad) + shift + 8,), MARK, device="cuda", dtype=getattr(torch, dtype))
    v = buf[shift:shift + rows * (n + pad)].view(rows, n + pad)[:, :n]
    v.copy_(put(a, dtype))
    return v


# ---- route ------------------------------------------------------------------------------------------------------------

ROUTES = [  # n, k, groups, keep, top
    (1, 1, 1, 1, 1), (2, 2, 1, 1, 1), (7, 3, 1, 1, 1), (8, 8, 1, 1, 1), (33, 2, 1, 1, 1), (64, 2, 1, 1, 1), (64, 64, 1, 1, 1),
    (65, 5, 1, 1, 1), (127, 8, 1, 1, 1), (129, 1, 1, 1, 1), (256, 8, 8, 4, 2), (257, 6, 1, 1, 1), (500, 16, 1, 1, 1),
    (513, 4, 1, 1, 1), (1000, 9, 5, 2, 2), (1023, 64, 33, 4, 1), (1024, 8, 64, 3, 2), (12, 2, 12, 5, 2), (12, 4, 3, 2, 1),
    (51, 9, 17, 6, 2), (6, 1, 2, 1, 2)]


def logits_for(rows, n, dtype, seed):
    r = np.random.default_rng(seed)
    l = (2.0 * r.normal(size=(rows, n))).astype(np.float32)
    low = {"float32": -3.4028235e38, "bfloat16": -3.3895314e38, "float16": -65504.0}[dtype]
    if rows > 8:
        l[1] = -np.inf                                      # a padded token
        l[2] = -np.inf
        l[2, n // 2] = 0.5                                  # one expert left
        l[3] = low                                          # masked with the lowest number: all alike
        l[4, :n // 2] = low
        l[5, ::3] = np.nan
        l[6] = np.round(l[6])                               # ties
        l[7, ::2] = -np.inf
        l[8, n - 1] = np.inf
    return rounded(l, dtype)


@pytest.mark.parametrize("n,k,groups,keep,top", ROUTES)
@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
def test_route(gpu, n, k, groups, keep, top, dtype):
    for rows in (1, 19):
        l = logits_for(rows, n, dtype, 100 * n + k)
        bias = (0.3 * np.random.default_rng(n).normal(size=n)).astype(np.float32)
        if n > 6:
            bias[3], bias[5] = -np.inf, np.nan
        for sigmoid in (False, True):
            for b in (None, bias):
                for renorm, scale in ((True, 1.0), (False, 2.5)):
                    print("case", rows, n, k, groups, keep, top, dtype, sigmoid, b is not None, renorm, flush=True)
                    x = strided(l, dtype, 3, 1) if sigmoid else put(l, dtype)
                    idx, val = gpu.topk_route_fwd(x, k, int(sigmoid), bias=None if b is None else put(b), groups=groups,
                                                  keep_groups=keep, group_top=top, renormalise=renorm, scale=scale)
                    want, weight = ref.route(l, k, sigmoid, b, groups, keep, top, renorm, scale)
                    got = host(idx)
                    assert got.dtype == np.int32 and np.array_equal(got, want), (got[:4], want[:4])
                    there = want >= 0
                    at = np.where(there, want, 0)
                    c = np.where(there, np.take_along_axis(np.nan_to_num(l, nan=0.0), at, 1), 0.0)
                    if sigmoid:
                        c = np.minimum(c, 0.0)
                    m = np.where(there, c, -np.inf).max(axis=1, keepdims=True)
                    if not renorm:
                        m = np.zeros_like(m) if sigmoid else np.nanmax(np.where(np.isnan(l), -np.inf, l), axis=1, keepdims=True)
                    with np.errstate(all="ignore"):
                        d = np.where(there & (c != m), np.abs(c - m), 0.0)
                        d = np.where(d > 200, 0.0, d)       # (exp of it is zero)
                    within(host(val), weight, (d + 56) * U * np.abs(weight) + 2.0 ** -126, "val")


@pytest.mark.parametrize("n,k", [(1, 1), (7, 3), (64, 2), (65, 8), (128, 8), (300, 16), (513, 5), (1024, 64)])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
def test_route_vjp(gpu, n, k, dtype):
    for rows in (1, 21):
        l = logits_for(rows, n, dtype, n + k)
        r = np.random.default_rng(k)
        t = r.normal(size=(rows, k)).astype(np.float32)
        idx = ref.route(l, k)[0]
        if rows > 12:
            idx[9] = -1
            idx[10, k // 2] = n                              # out of range: an empty place
            idx[11] = idx[11, 0]                             # the same expert in every place
            t[2, 1:] = np.nan                                # (its places are empty)
        for sigmoid in (False, True):
            for renorm, scale in ((True, 1.0), (False, 2.5)):
                print("case", rows, n, k, dtype, sigmoid, renorm, flush=True)
                x = strided(l, dtype, 5, 2) if renorm else put(l, dtype)
                got = host(gpu.topk_route_vjp(x, put(idx, "int32"), put(t), int(sigmoid), renormalise=renorm, scale=scale))
                want = ref.route_vjp(l, idx, t, sigmoid, renorm, scale)
                # every term is a product of weights, each off by (D + 56) u, D < 30 for those that count, and a sum over
                # k choices; the terms' size is bounded by that of the gradient with |t| and signs that add up
                p, lg = ref.scores(l, sigmoid), ref.log_scores(l, sigmoid)
                there = (idx >= 0) & (idx < n)
                at = np.where(there, idx, 0)
                there = there & (np.take_along_axis(lg, at, 1) > -np.inf)
                w = np.where(there, np.take_along_axis(p, at, 1), 0.0)
                if renorm:
                    c = np.where(there, np.take_along_axis(lg, at, 1), -np.inf)
                    m = c.max(axis=1, keepdims=True)
                    with np.errstate(all="ignore"):
                        w = np.where(there, np.where(c == m, 1.0, np.exp(c - m)), 0.0)
                    z = w.sum(axis=1, keepdims=True)
                    w = w / np.where(z == 0, 1, z)
                a = np.where(there & (w > 0), np.abs(t), 0.0)
                mean = (w * a).sum(axis=1, keepdims=True)
                size = np.zeros_like(p)
                np.add.at(size, (np.arange(rows)[:, None], at), np.where(there, w * (a + mean), 0.0))
                if not renorm and not sigmoid:
                    size += p * mean
                # the reference itself: renormalised softmax subtracts k products v s of float64 from every entry, whose
                # exact sum is zero for experts that are not chosen: k products of at most 2 max|t|, rounded twice each
                own = 4 * k * 2.0 ** -53 * np.abs(np.nan_to_num(t)).max() * scale
                within(got, want, 2 * (30 + 56 + k) * U * scale * size + HALF[dtype] * np.abs(want) + TINY[dtype] + 2.0 ** -126
                       + own, "grad")


def test_route_rows_of_a_broadcast(gpu):
    """One row of logits for all tokens (stride 0)."""
    import torch
    l = put(np.random.default_rng(3).normal(size=(1, 40)))
    idx, val = gpu.topk_route_fwd(l.expand(6, 40), 3)
    one, w = gpu.topk_route_fwd(l, 3)
    assert torch.equal(idx, one.expand(6, 3)) and torch.equal(val, w.expand(6, 3))


# ---- places -----------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("rows,k,n", [(0, 2, 5), (1, 1, 1), (1, 8, 64), (63, 2, 64), (64, 2, 64), (513, 3, 7), (1025, 2, 1024),
                                      (2048, 1, 2), (2049, 1, 3), (5000, 4, 100), (3001, 7, 1000), (40000, 2, 33)])
@pytest.mark.parametrize("kind", ["spread", "one", "padded", "none"])
def test_places(gpu, rows, k, n, kind):
    r = np.random.default_rng(rows + n)
    idx = r.integers(0, n, size=(rows, k)).astype(np.int32)
    if kind == "one":
        idx[:] = n - 1
    elif kind == "padded":
        idx[r.random(rows) < 0.3] = -1
        if rows > 4:
            idx[3, 0], idx[4, k - 1], idx[2, 0] = n, 2 ** 31 - 1, -2 ** 31
    elif kind == "none":
        idx[:] = -1
    for capacity in (0, 1, 1 + rows * k // (2 * n), 2 ** 40):
        print("case", rows, k, n, kind, capacity, flush=True)
        want = ref.places(idx, n, min(capacity, 2 ** 31))
        for got, w, name in zip(gpu.topk_expert_map(put(idx, "int32"), n, capacity=capacity), want,
                                ("slot", "source", "offset", "load")):
            assert np.array_equal(host(got), w), name


# ---- products ---------------------------------------------------------------------------------------------------------

PRODUCTS = [  # rows, k, n, h, ho
    (1, 1, 1, 1, 1), (1, 2, 4, 16, 8), (5, 2, 3, 33, 17), (40, 2, 4, 64, 64), (64, 2, 2, 128, 128), (70, 3, 5, 100, 260),
    (300, 1, 2, 136, 72), (130, 2, 1, 31, 129), (9, 4, 40, 256, 128), (260, 2, 3, 72, 264),
    (700, 2, 3, 328, 520), (20, 2, 3, 9, 15), (25, 1, 2, 8, 8), (50, 2, 2, 13, 67), (33, 2, 3, 23, 71), (150, 2, 2, 135, 193),
    (90, 1, 2, 4, 5), (60, 2, 3, 70, 3)]


def product_case(rows, k, n, h, ho, dtype, gather, wide, seed):
    r = np.random.default_rng(seed)
    idx = np.stack([r.permutation(n)[:k] if n >= k else r.integers(0, n, k) for _ in range(rows)]).astype(np.int32)
    idx[r.random(rows) < 0.15] = -1
    if n > 2:
        idx[idx == 1] = 0                                    # an expert without places
    slot, source, offset, _ = ref.places(idx, n)
    m = rows if gather else rows * k
    x, w = rounded(r.normal(size=(m, h)), dtype), rounded(r.normal(size=(n, ho, h)), dtype)
    t = rounded(r.normal(size=(rows * k, ho)), dtype)
    wd = put(w, dtype) if not wide else put(w.transpose(0, 2, 1), dtype).transpose(1, 2)
    return x, w, t, wd, slot, source if gather else None, offset


@pytest.mark.parametrize("rows,k,n,h,ho", PRODUCTS)
@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
def test_products(gpu, rows, k, n, h, ho, dtype):
    import torch
    for gather in (True, False):
        for transposed in (False, True):
            for shift in (0, 1):
                print("case", rows, k, n, h, ho, dtype, gather, transposed, shift, flush=True)
                x, w, t, wd, _, source, offset = product_case(rows, k, n, h, ho, dtype, gather, transposed, rows + h)
                xd = strided(x, dtype, 3, 1) if shift else put(x, dtype)
                td = strided(t, dtype, 1, 1) if shift else put(t, dtype)
                sd = None if source is None else put(source, "int32")
                od = put(offset, "int32")
                out = torch.full((rows * k, ho), MARK, device="cuda", dtype=xd.dtype)
                assert gpu.topk_expert_product_fwd(xd, wd, od, source=sd, k=k, out=out) is out
                want, size = ref.product(x, w, offset, source, k)
                end = offset[-1]
                got = host(out)
                assert (got[end:] == MARK).all(), "a row behind the last place was written"
                within(got[:end], want[:end], (h + 2) * 2 * U * size[:end] + HALF[dtype] * np.abs(want[:end]) + TINY[dtype], "out")
                dx = torch.full((rows * k, h), MARK, device="cuda", dtype=xd.dtype)
                dxg, dw = gpu.topk_expert_product_vjp(xd, wd, od, td, source=sd, k=k, dx_out=dx)
                assert dxg is dx and dw.shape == wd.shape and dw.stride() == wd.stride()
                wx, ww, sx, sw = ref.product_vjp(x, w, offset, source, k, t)
                got = host(dx)
                assert (got[end:] == MARK).all(), "a row behind the last place was written"
                within(got[:end], wx[:end], (ho + 2) * 2 * U * sx[:end] + HALF[dtype] * np.abs(wx[:end]) + TINY[dtype], "dx")
                most = max(1, int(np.diff(offset).max()))
                within(host(dw), ww, (most + 2) * 2 * U * sw + HALF[dtype] * np.abs(ww) + TINY[dtype], "dw")
                only, none = gpu.topk_expert_product_vjp(xd, wd, od, td, source=sd, k=k, want_w=False)
                assert none is None and torch.equal(only[:end], dx[:end])
                none, only = gpu.topk_expert_product_vjp(xd, wd, od, td, source=sd, k=k, want_x=False)
                assert none is None and torch.equal(only, dw)


@pytest.mark.parametrize("rows,k,n,h,ho", [(1500, 2, 24, 1032, 1040), (1500, 2, 24, 1033, 1047), (1500, 2, 24, 1034, 1042),
                                           (2100, 1, 6, 2056, 2048), (700, 3, 5, 131, 1411)])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
def test_large_products(gpu, rows, k, n, h, ho, dtype):
    """Sizes of the larger tiles, experts of very different loads; the sums in float64, expert by expert."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(rows + h)
    dt = getattr(torch, dtype)
    liked = 1.5 * torch.randn((1, n), generator=g, device="cuda")
    idx = (torch.randn((rows, n), generator=g, device="cuda") + liked).topk(k, dim=1).indices.to(torch.int32).contiguous()
    idx[torch.rand(rows, generator=g, device="cuda") < 0.1] = -1
    _, source, offset, _ = gpu.topk_expert_map(idx, n)
    x = torch.randn((rows, h), generator=g, device="cuda").to(dt)
    t = torch.randn((rows * k, ho), generator=g, device="cuda").to(dt)
    w = torch.randn((n, ho, h), generator=g, device="cuda").to(dt)
    at = offset.tolist()
    for transposed in (False, True):
        print("case", rows, k, n, h, ho, dtype, transposed, flush=True)
        wd = w.transpose(1, 2).contiguous().transpose(1, 2) if transposed else w
        out = torch.full((rows * k, ho), MARK, device="cuda", dtype=dt)
        gpu.topk_expert_product_fwd(x, wd, offset, source=source, k=k, out=out)
        dx = torch.full((rows * k, h), MARK, device="cuda", dtype=dt)
        _, dw = gpu.topk_expert_product_vjp(x, wd, offset, t, source=source, k=k, dx_out=dx)
        assert (out[at[n]:] == MARK).all() and (dx[at[n]:] == MARK).all()
        for e in range(n):
            part = slice(at[e], at[e + 1])
            xe, te, we = x[(source[part] // k).long()].double(), t[part].double(), w[e].double()
            for have, a, b, terms, name in ((out[part], xe, we.t().contiguous(), h, "out"), (dx[part], te, we, ho, "dx"),
                                            (dw[e], te.t().contiguous(), xe, at[e + 1] - at[e], "dw")):
                want = host(a @ b)
                size = host(a.abs() @ b.abs())
                within(host(have), want, (terms + 2) * 2 * U * size + HALF[dtype] * np.abs(want) + TINY[dtype], (name, e))


def test_products_of_no_places(gpu):
    import torch
    w = torch.randn((3, 5, 4), device="cuda")
    x = torch.empty((0, 4), device="cuda")
    off = torch.zeros(4, dtype=torch.int32, device="cuda")
    assert gpu.topk_expert_product_fwd(x, w, off).shape == (0, 5)
    dx, dw = gpu.topk_expert_product_vjp(x, w, off, torch.empty((0, 5), device="cuda"))
    assert dx.shape == (0, 4) and (dw == 0).all()


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_product_with_lists_out_of_range(gpu, dtype):
    """Sources outside the rows give zeros; offsets outside the places are cut off."""
    import torch
    r = np.random.default_rng(4)
    x, w = rounded(r.normal(size=(6, 16)), dtype), rounded(r.normal(size=(2, 8, 16)), dtype)
    source = np.array([0, 3, -5, 2 ** 31 - 1, 12, 11, 7, 4], np.int32)           # k = 2: rows 0, 1, -, -, -, 5, 3, 2
    offset = np.array([0, 5, 8], np.int32)
    t = rounded(r.normal(size=(8, 8)), dtype)
    xs = np.zeros((8, 16))
    for s, row in ((0, 0), (1, 1), (5, 5), (6, 3), (7, 2)):
        xs[s] = x[row]
    out = host(gpu.topk_expert_product_fwd(put(x, dtype), put(w, dtype), put(offset, "int32"), put(source, "int32"), 2))
    want, size = ref.product(xs, w, offset, None, 1)
    within(out, want, 18 * 2 * U * size + HALF[dtype] * np.abs(want), "out")
    _, dw = gpu.topk_expert_product_vjp(put(x, dtype), put(w, dtype), put(offset, "int32"), put(t, dtype),
                                        put(source, "int32"), 2)
    _, ww, _, sw = ref.product_vjp(xs, w, offset, None, 1, t)
    within(host(dw), ww, 7 * 2 * U * sw + HALF[dtype] * np.abs(ww), "dw")
    for bad in ([-7, 5, 100], [0, 5, 3], [2 ** 31 - 1, 0, 8], [-2 ** 31, -2 ** 31, 2 ** 31 - 1]):
        gpu.topk_expert_product_fwd(put(x, dtype), put(w, dtype), put(np.array(bad, np.int32), "int32"), put(source, "int32"), 2)
        gpu.topk_expert_product_vjp(put(x, dtype), put(w, dtype), put(np.array(bad, np.int32), "int32"), put(t, dtype),
                                    put(source, "int32"), 2)
    torch.cuda.synchronize()


# ---- combine ----------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("rows,k,h", [(1, 1, 1), (3, 2, 7), (17, 3, 64), (5, 8, 255), (40, 2, 1024), (9, 4, 2049), (2, 1, 9000),
                                      (33, 11, 40)])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
def test_combine(gpu, rows, k, h, dtype):
    import torch
    r = np.random.default_rng(rows * h)
    slots = rows * k + 2
    slot = r.permutation(slots)[:rows * k].reshape(rows, k).astype(np.int32)
    if rows > 2:
        slot[0] = -1
        slot[1, k - 1], slot[2, 0] = slots, -2 ** 31
    y, g = rounded(r.normal(size=(slots, h)), dtype), rounded(r.normal(size=(rows, h)), dtype)
    val = r.normal(size=(rows, k)).astype(np.float32)
    if rows > 2:
        val[0] = np.nan                                      # weights of empty places count for nothing
    there = (slot >= 0) & (slot < slots)
    v64 = np.where(there, val, 0.0).astype(np.float64)
    unused = np.setdiff1d(np.arange(slots), slot[there])
    for shift in (0, 1):
        for weights in (True, False):
            print("case", rows, k, h, dtype, shift, weights, flush=True)
            yd = strided(y, dtype, 3, 1) if shift else put(y, dtype)
            gd = strided(g, dtype, 1, 3) if shift else put(g, dtype)
            vd, w = (put(val), v64) if weights else (None, np.ones_like(v64))
            want, size = ref.combine(y, slot, w)
            within(host(gpu.topk_combine_fwd(yd, put(slot, "int32"), vd)), want,
                   (k + 1) * U * size + HALF[dtype] * np.abs(want) + TINY[dtype], "out")
            dy = torch.full((slots, h), MARK, device="cuda", dtype=yd.dtype)
            dyg, dval = gpu.topk_combine_vjp(yd, put(slot, "int32"), vd, gd, dy_out=dy)
            wy, wv, sv = ref.combine_vjp(y, slot, w, g)
            got = host(dyg)
            assert (got[unused] == MARK).all(), "a row that no pair names was written"
            used = np.setdiff1d(np.arange(slots), unused)
            within(got[used], wy[used], (U + HALF[dtype]) * np.abs(wy[used]) + TINY[dtype], "dy")
            if weights:
                within(host(dval), wv, (h + 1) * U * sv, "dval")
            else:
                assert dval is None


# ---- together ---------------------------------------------------------------------------------------------------------

def layer(gpu, l, x, w1, w2, g, k, n, route):
    """Two products with a rectifier between, and every gradient: as a training step makes the calls."""
    import torch
    idx, val = route(l)
    slot, source, offset, load = gpu.topk_expert_map(idx, n)
    u = gpu.topk_expert_product_fwd(x, w1, offset, source=source, k=k)
    a = torch.relu(u)
    y = gpu.topk_expert_product_fwd(a, w2, offset)
    out = gpu.topk_combine_fwd(y, slot, val)
    dy, dval = gpu.topk_combine_vjp(y, slot, val, g)
    da, dw2 = gpu.topk_expert_product_vjp(a, w2, offset, dy)
    du = da * (u > 0)
    dxs, dw1 = gpu.topk_expert_product_vjp(x, w1, offset, du, source=source, k=k)
    return idx, val, out, dval, gpu.topk_combine_fwd(dxs, slot), dw1, dw2, load


def dense(l, x, w1, w2, g, idx, sigmoid):
    """The same in float64 with every expert for every token, gradients by autograd."""
    import torch
    t = [torch.from_numpy(np.array(a, np.float64)).requires_grad_() for a in (l, x, w1, w2)]
    s = torch.sigmoid(t[0]) if sigmoid else torch.softmax(t[0], dim=1)
    there = torch.from_numpy(idx >= 0)
    w = torch.where(there, s.gather(1, torch.from_numpy(np.where(idx < 0, 0, idx)).long()), 0.0)
    w = w / w.sum(dim=1, keepdim=True)
    per = torch.stack([torch.relu(t[1] @ t[2][e].t()) @ t[3][e].t() for e in range(w1.shape[0])], dim=1)
    full = torch.zeros(l.shape, dtype=torch.float64).scatter_add(1, torch.from_numpy(np.where(idx < 0, 0, idx)).long(), w)
    out = (full.unsqueeze(2) * per).sum(dim=1)
    (out * torch.from_numpy(g)).sum().backward()
    return [out.detach().numpy()] + [a.grad.numpy() for a in t]


@pytest.mark.parametrize("dtype,bar", [("float32", 2e-5), ("bfloat16", 4e-2), ("float16", 5e-3)])
@pytest.mark.parametrize("sigmoid", [False, True])
def test_layer(gpu, dtype, bar, sigmoid):
    """Relative to the largest value of each array: four roundings to the type on the way (8 half steps leave room for the
    growth through the second product), and for float32 sums of 96 terms."""
    rows, n, k, h, f = 150, 9, 3, 64, 96
    r = np.random.default_rng(8)
    l = r.normal(size=(rows, n)).astype(np.float32)
    x, g = rounded(r.normal(size=(rows, h)), dtype), rounded(r.normal(size=(rows, h)), dtype)
    w1, w2 = rounded(r.normal(size=(n, f, h)) / 8, dtype), rounded(r.normal(size=(n, h, f)) / 10, dtype)
    got = layer(gpu, put(l), put(x, dtype), put(w1, dtype), put(w2, dtype), put(g, dtype), k, n,
                lambda v: gpu.topk_route_fwd(v, k, int(sigmoid)))
    idx = host(got[0])
    dl = gpu.topk_route_vjp(put(l), got[0], got[3], int(sigmoid))
    want = dense(l, x, w1, w2, g, idx, sigmoid)
    for have, w, name in ((got[2], want[0], "out"), (dl, want[1], "dlogits"), (got[4], want[2], "dx"), (got[5], want[3], "dw1"),
                          (got[6], want[4], "dw2")):
        within(host(have), w, bar * np.abs(w).max(), name)


def test_layer_behind_the_relaxed_router(gpu):
    """The lists of topk_mask_sparse_fwd go the same way; their weights' gradient goes through topk_mask_vjp."""
    import torch
    rows, n, h, f, width = 90, 12, 32, 48, 6
    r = np.random.default_rng(9)
    l = r.normal(size=(rows, n)).astype(np.float32)
    x, g = r.normal(size=(rows, h)).astype(np.float32), r.normal(size=(rows, h)).astype(np.float32)
    w1, w2 = (r.normal(size=(n, f, h)) / 6).astype(np.float32), (r.normal(size=(n, h, f)) / 7).astype(np.float32)
    ld = put(l)
    idx, val, out, dval, dx, dw1, dw2, load = layer(gpu, ld, put(x), put(w1), put(w2), put(g), width, n,
                                                    lambda v: gpu.topk_mask_sparse_fwd(v, 2, 2.0, 0.5, width)[:2])
    mask = gpu.topk_mask_fwd(ld, 2, 2.0, 0.5)
    assert int((mask > 0).sum(dim=1).max()) <= width and torch.equal(load, (mask > 0).sum(dim=0).to(torch.int32))
    cot = torch.zeros((rows, n), device="cuda").scatter_add_(1, idx.clamp(min=0).long(), torch.where(idx >= 0, dval, 0.0))
    _, dl = gpu.topk_mask_vjp(ld, cot, 2, 2.0, 0.5)
    t = [torch.from_numpy(a.astype(np.float64)).requires_grad_() for a in (host(mask), x, w1, w2)]
    per = torch.stack([torch.relu(t[1] @ t[2][e].t()) @ t[3][e].t() for e in range(n)], dim=1)
    ref_out = (t[0].unsqueeze(2) * per).sum(dim=1)
    (ref_out * torch.from_numpy(g.astype(np.float64))).sum().backward()
    for have, want, name in ((out, ref_out, "out"), (dx, t[1].grad, "dx"), (dw1, t[2].grad, "dw1"), (dw2, t[3].grad, "dw2")):
        w = want.detach().numpy()
        within(host(have), w, 2e-5 * np.abs(w).max(), name)
    # the cotangent of the mask where the mask is not zero
    w = np.where(host(mask) > 0, t[0].grad.numpy(), 0.0)
    within(host(cot), w, 2e-5 * np.abs(w).max(), "dmask")
    assert torch.isfinite(dl).all()


# ---- graphs, streams, refusals ----------------------------------------------------------------------------------------

def test_layer_captured_and_replayed(gpu):
    """Two graphs over the same inputs, replayed in turn with new contents and eager work between; every replay against the
    eager calls."""
    import torch
    rows, n, k, h, f = 3000, 16, 2, 64, 32                   # (a map of several workgroups)
    gen = torch.Generator(device="cuda").manual_seed(1)

    def randn(*shape):
        return torch.randn(shape, generator=gen, device="cuda")
    l, x, g = randn(rows, n), randn(rows, h).bfloat16(), randn(rows, h).bfloat16()
    w1, w2 = (randn(n, f, h) / 8).bfloat16(), (randn(n, h, f) / 6).bfloat16()

    def step():
        r = layer(gpu, l, x, w1, w2, g, k, n, lambda v: gpu.topk_route_fwd(v, k))
        return r + (gpu.topk_route_vjp(l, r[0], r[3]),)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graphs, outs = [], []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(step())
        graphs.append(graph)
    for turn in range(4):
        for t in (l, x, g):
            t.copy_(randn(*t.shape))
        graphs[turn % 2].replay()
        torch.cuda.synchronize()
        eager = step()
        torch.cuda.synchronize()
        for a, b in zip(outs[turn % 2], eager):
            assert torch.equal(a, b), turn


def test_given_stream(gpu):
    """A stream that is passed in takes the work, as an object or as a handle."""
    import torch
    l = torch.randn((500, 24), device="cuda")
    y = torch.randn((1000, 40), device="cuda")
    idx, val = gpu.topk_route_fwd(l, 2)
    slot, source, offset, load = gpu.topk_expert_map(idx, 24)
    want = gpu.topk_combine_fwd(y, slot, val)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    for given in (s, int(s.cuda_stream)):
        busy = torch.randn((2048, 2048), device="cuda")
        l2 = torch.zeros_like(l)
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            for _ in range(20):
                busy = busy @ busy / 50.0
            l2.copy_(l)                                      # in order behind the products on s
        i2, v2 = gpu.topk_route_fwd(l2, 2, stream=given)
        m2 = gpu.topk_expert_map(i2, 24, stream=given)
        o2 = gpu.topk_combine_fwd(y, m2[0], v2, stream=given)
        s.synchronize()
        assert torch.equal(i2, idx) and torch.equal(v2, val) and torch.equal(o2, want)
        for a, b in zip(m2, (slot, source, offset, load)):
            assert torch.equal(a, b)


def test_calls_on_two_streams(gpu):
    """Maps of several workgroups at the same time: they share no scratch."""
    import torch
    a = torch.randint(0, 64, (50000, 2), dtype=torch.int32, device="cuda")
    b = torch.randint(0, 64, (50000, 2), dtype=torch.int32, device="cuda")
    want = [gpu.topk_expert_map(i, 64) for i in (a, b)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(10):
        for i, s in enumerate(streams):
            got[i].append(gpu.topk_expert_map((a, b)[i], 64, stream=s))
    torch.cuda.synchronize()
    for i in range(2):
        for r in got[i]:
            assert all(torch.equal(p, q) for p, q in zip(r, want[i]))


def test_refusals(gpu):
    import torch
    f, i = torch.randn((8, 16), device="cuda"), torch.zeros((8, 2), dtype=torch.int32, device="cuda")
    w, off = torch.randn((3, 5, 16), device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
    v, src = torch.ones((8, 2), device="cuda"), torch.zeros(16, dtype=torch.int32, device="cuda")
    t = torch.randn((16, 5), device="cuda")
    bad = [lambda: gpu.topk_route_fwd(f.double(), 2), lambda: gpu.topk_route_fwd(f[0], 2), lambda: gpu.topk_route_fwd(f, 17),
           lambda: gpu.topk_route_fwd(f, 0), lambda: gpu.topk_route_fwd(f, -1), lambda: gpu.topk_route_fwd(f.t(), 2),
           lambda: gpu.topk_route_fwd(f, 2, 3), lambda: gpu.topk_route_fwd(f, 2, bias=f[0, :8]),
           lambda: gpu.topk_route_fwd(f, 2, bias=f[0].half()), lambda: gpu.topk_route_fwd(f, 2, groups=3),
           lambda: gpu.topk_route_fwd(f, 2, idx_out=i.long()), lambda: gpu.topk_route_fwd(f, 2, val_out=f[:, :2]),
           lambda: gpu.topk_route_fwd(f, 2, idx_out=i, val_out=i.view(torch.float32)),
           lambda: gpu.topk_route_fwd(torch.randn((2, 1025), device="cuda"), 2),
           lambda: gpu.topk_route_vjp(f, i.long(), v), lambda: gpu.topk_route_vjp(f, i, v[:4]),
           lambda: gpu.topk_route_vjp(f, i, v.half()), lambda: gpu.topk_route_vjp(f, i, v, grad_out=f),
           lambda: gpu.topk_expert_map(i.long(), 3), lambda: gpu.topk_expert_map(i, 0), lambda: gpu.topk_expert_map(i, 1025),
           lambda: gpu.topk_expert_map(i, 3, capacity=-1), lambda: gpu.topk_expert_map(i[:, :1], 3),
           lambda: gpu.topk_expert_map(i, 3, slot_out=i), lambda: gpu.topk_expert_map(i, 3, load_out=off),
           lambda: gpu.topk_expert_product_fwd(f, w.half(), off), lambda: gpu.topk_expert_product_fwd(f, w[:, :, ::2], off),
           lambda: gpu.topk_expert_product_fwd(f[:, ::2], w[:, :, ::2], off), lambda: gpu.topk_expert_product_fwd(f, w, off[:3]),
           lambda: gpu.topk_expert_product_fwd(f, w, off, source=src.long()),
           lambda: gpu.topk_expert_product_fwd(f, w, off, source=src, k=0),
           lambda: gpu.topk_expert_product_fwd(f, w, off, out=t), lambda: gpu.topk_expert_product_fwd(f, w[0], off),
           lambda: gpu.topk_expert_product_vjp(f, w, off, t), lambda: gpu.topk_expert_product_vjp(f, w, off, t[:8].half()),
           lambda: gpu.topk_expert_product_vjp(f, w, off, t[:8], dx_out=f),
           lambda: gpu.topk_expert_product_vjp(f, w, off, t[:8], dw_out=w),
           lambda: gpu.topk_expert_product_vjp(f, w.transpose(1, 2).contiguous().transpose(1, 2), off, t[:8],
                                               dw_out=torch.empty_like(w).contiguous()),
           lambda: gpu.topk_combine_fwd(f, i.long()), lambda: gpu.topk_combine_fwd(f, i, v.half()),
           lambda: gpu.topk_combine_fwd(f, i, v[:4]), lambda: gpu.topk_combine_fwd(f, i, v, out=f),
           lambda: gpu.topk_combine_vjp(f, i, v, f[:4]), lambda: gpu.topk_combine_vjp(f, i, v, f.half()),
           lambda: gpu.topk_combine_vjp(f, i, v, f.clone(), dy_out=f), lambda: gpu.topk_combine_vjp(f, i, v, f, dval_out=v)]
    for j, call in enumerate(bad):
        with pytest.raises(gpu.TopkError):
            call()
            raise AssertionError(f"call {j} was not refused")
    torch.cuda.synchronize()


def test_native_step_and_python_agree(gpu):
    """Results, errors and returned objects of the binding's native step against the Python code behind it."""
    import torch
    from tests.test_gpu_native_call import both as compare
    assert gpu._call is not None, "the native call path was not built"

    def both(f):
        def tensors():
            r = f()
            r = r if isinstance(r, tuple) else (r,)
            return tuple(t for t in r if t is not None) + (sum(t is None for t in r),)
        return compare(gpu, tensors)
    g = torch.Generator(device="cuda").manual_seed(5)
    for dtype in (torch.float32, torch.bfloat16, torch.float16):
        l = torch.randn((70, 24), generator=g, device="cuda").to(dtype)
        wide = torch.randn((70, 30), generator=g, device="cuda").to(dtype)[:, 3:27]
        bias, t = torch.randn(24, generator=g, device="cuda"), torch.randn((70, 2), generator=g, device="cuda")
        for x in (l, wide, l[:0], l.t().contiguous().t()):
            both(lambda: gpu.topk_route_fwd(x, 2))
            both(lambda: gpu.topk_route_fwd(x, 3, gpu.TOPK_SCORE_SIGMOID, bias=bias, groups=4, keep_groups=2, group_top=2,
                                            renormalise=False, scale=2))
        idx, val = gpu.topk_route_fwd(l, 2)
        both(lambda: gpu.topk_route_vjp(wide, idx, t, renormalise=False))
        both(lambda: gpu.topk_route_vjp(l, idx, t, 1, scale=0.5))
        both(lambda: gpu.topk_expert_map(idx, 24))
        both(lambda: gpu.topk_expert_map(idx.expand(70, 2)[:0], 24, capacity=1))
        both(lambda: gpu.topk_expert_map(idx.repeat(100, 1), 24, capacity=7))
        slot, source, offset, load = gpu.topk_expert_map(idx, 24)
        x, w = torch.randn((70, 16), generator=g, device="cuda").to(dtype), torch.randn((24, 8, 16), generator=g, device="cuda").to(dtype)
        c = torch.randn((140, 8), generator=g, device="cuda").to(dtype)
        for u in (w, w.transpose(1, 2).contiguous().transpose(1, 2), w[:, :, :1], w[:, :1]):
            xu = x[:, :u.shape[2]]
            both(lambda: gpu.topk_expert_product_fwd(xu, u, offset, source, 2))
            cu = c[:, :u.shape[1]]
            for want in ((True, True), (True, False), (False, True), (False, False)):
                both(lambda: gpu.topk_expert_product_vjp(xu, u, offset, cu, source, 2, *want))
        y = gpu.topk_expert_product_fwd(x, w, offset, source, 2)
        out = torch.randn((70, 8), generator=g, device="cuda").to(dtype)
        dy = torch.zeros_like(y)
        both(lambda: gpu.topk_combine_fwd(y, slot, val))
        both(lambda: gpu.topk_combine_fwd(y, slot))
        both(lambda: gpu.topk_combine_vjp(y, slot, val, out))
        both(lambda: gpu.topk_combine_vjp(y, slot, None, out, dy_out=dy))
        assert gpu.topk_combine_vjp(y, slot, val, out, dy_out=dy)[0] is dy
        for bad in (lambda: gpu.topk_route_fwd(l, 25), lambda: gpu.topk_route_fwd(l, -1), lambda: gpu.topk_route_fwd(l, 2, 7),
                    lambda: gpu.topk_route_fwd(l, 2, groups=5), lambda: gpu.topk_route_fwd(l.cpu(), 2),
                    lambda: gpu.topk_route_fwd(l, 2, bias=bias[:5]), lambda: gpu.topk_route_vjp(l, idx[:5], t),
                    lambda: gpu.topk_expert_map(idx, 0), lambda: gpu.topk_expert_map(idx.long(), 24),
                    lambda: gpu.topk_expert_product_fwd(x, w, offset[:3], source, 2),
                    lambda: gpu.topk_expert_product_fwd(x, w, offset, source, 0),
                    lambda: gpu.topk_expert_product_vjp(x, w, offset, c[:5], source, 2), lambda: gpu.topk_combine_fwd(y, slot, val[:4]),
                    lambda: gpu.topk_combine_vjp(y, slot, val, out, dy_out=y), lambda: gpu.topk_combine_vjp(y, slot, val, out[:5])):
            r = compare(gpu, bad)
            assert isinstance(r[0], type) and issubclass(r[0], gpu.TopkError), r


# the zeros of an expert without places: blocks of any size, so of any alignment in memory, before and behind others
@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("h,ho", [(1, 1), (3, 5), (129, 7), (131, 257), (256, 520)])
def test_weight_gradient_of_experts_without_places(gpu, h, ho, dtype):
    import torch
    t = getattr(torch, dtype)
    counts = [0, 0, 2, 0, 1, 0]
    off = torch.tensor([0] + list(np.cumsum(counts)), dtype=torch.int32, device="cuda")
    x = torch.randn((3, h), device="cuda").to(t)
    ct = torch.randn((3, ho), device="cuda").to(t)
    for transposed in (False, True):
        w = torch.randn((6, h, ho) if transposed else (6, ho, h), device="cuda").to(t)
        w = w.transpose(1, 2) if transposed else w
        dw = torch.full((6, h, ho) if transposed else (6, ho, h), 7.0, device="cuda", dtype=t)
        dw = dw.transpose(1, 2) if transposed else dw
        _, got = gpu.topk_expert_product_vjp(x, w, off, ct, want_x=False, dw_out=dw)
        assert got is dw
        at = 0
        for e, c in enumerate(counts):
            if c == 0:
                assert torch.all(dw[e] == 0), (e, transposed)
            else:
                want = ct[at:at + c].cpu().double().t() @ x[at:at + c].cpu().double()
                # two roundings of products and one of their sum, one of the output (2^-25 for a subnormal float16)
                room = torch.finfo(t).eps / 2 * want.abs() + 3 * 2.0 ** -24 * (ct[at:at + c].cpu().double().abs().t() @
                                                                               x[at:at + c].cpu().double().abs())
                assert torch.all((dw[e].cpu().double() - want).abs() <= room + 2.0 ** -24), (e, transposed)
            at += c


# scores that float32 cannot tell apart, in runs of `run` neighbours of the order that end before, at and behind the k-th place
@pytest.mark.parametrize("n,k", [(6, 5), (40, 5), (64, 64), (200, 9), (1000, 64)])
@pytest.mark.parametrize("run", [1, 2, 3, 4, 1000])
def test_route_of_scores_that_cross_in_float32(gpu, n, k, run):
    r = np.random.default_rng(n + run)
    for sigmoid in (False, True):
        l = r.normal(size=(24, n)).astype(np.float32)
        l[1:] = l[0]                                        # neighbours differ by roundings of the logits and the bias
        for row in range(1, 24):
            at = r.integers(0, n, size=3)
            l[row, at] = np.nextafter(l[row, at], np.float32(9.0) * (-1) ** row)
        for start in range(min(run, 5)):
            rank = np.empty(n, np.int64)
            rank[r.permutation(n)] = (np.arange(n) + start) // run
            bias = (0.9 - 0.01 * rank - ref.scores(l[:1], sigmoid)[0]).astype(np.float32)
            want = ref.route(l, k, sigmoid, bias)[0]
            idx, _ = gpu.topk_route_fwd(put(l), k, int(sigmoid), bias=put(bias))
            assert np.array_equal(host(idx), want), (sigmoid, start)
        ties = np.round(l * 4) / 4
        idx, _ = gpu.topk_route_fwd(put(ties), k, int(sigmoid), bias=put(np.zeros(n)))
        assert np.array_equal(host(idx), ref.route(ties, k, sigmoid, np.zeros(n))[0]), "ties"


def test_calls_of_more_rows_than_a_launch_takes(gpu):
    """Rows at both ends of a call that is cut into several launches."""
    import torch
    rows = (1 << 25) + 3
    at = torch.tensor([0, 1, (1 << 23) - 1, 1 << 23, (1 << 25) - 1, 1 << 25, rows - 1], device="cuda")
    l = torch.randn((rows, 2), device="cuda").half()
    idx, val = gpu.topk_route_fwd(l, 1, renormalise=False)
    want_idx, want_val = gpu.topk_route_fwd(l[at], 1, renormalise=False)
    assert torch.equal(idx[at], want_idx) and torch.equal(val[at], want_val)
    assert torch.equal(idx[:, 0], (l[:, 1] > l[:, 0]).int())
    t = torch.randn((rows, 1), device="cuda")
    grad = gpu.topk_route_vjp(l, idx, t, renormalise=False)
    assert torch.equal(grad[at], gpu.topk_route_vjp(l[at], idx[at], t[at].contiguous(), renormalise=False))
    # the two cancel: an output's rounding each, and float32 roundings of terms up to |t|
    assert (grad.float().sum(dim=1).abs() <= 2.0 ** -11 * grad.float().abs().sum(dim=1) + 2.0 ** -21 * t.abs()[:, 0] + 2.0 ** -24).all()
    slot = torch.arange(rows - 1, -1, -1, device="cuda", dtype=torch.int32)[:, None].contiguous()
    out = gpu.topk_combine_fwd(l, slot, t)
    # one product, rounded to float32 and to float16, or (a multiplication that ends in float16) to float16 alone
    def product(got, a):
        exact = a.double() * t.double()
        assert ((got.double() - exact).abs() <= (2.0 ** -11 + 2.0 ** -23) * exact.abs() + 2.0 ** -25).all()
    product(out, l.flip(0))
    dy, dval = gpu.topk_combine_vjp(l, slot, t, out)
    product(dy.flip(0), out)
    want = (out.double() * l.flip(0).double()).sum(dim=1, keepdim=True)
    # two products, exact in float32, and their sum
    assert ((dval.double() - want).abs() <= 2.0 ** -23 * (out.double() * l.flip(0).double()).abs().sum(dim=1, keepdim=True)).all()


def test_refusals_of_scales_and_counts(gpu):
    import ctypes
    import torch
    l = torch.randn((4, 8), device="cuda")
    with pytest.raises(gpu.TopkError):
        gpu.topk_route_fwd(l, 2, scale=1e300)               # infinite in float32
    with pytest.raises(gpu.TopkError):
        gpu.topk_route_vjp(l, torch.zeros((4, 1), dtype=torch.int32, device="cuda"), l[:, :1].contiguous(), scale=-1e39)
    lib, one = gpu.load(), ctypes.c_void_p(256)             # (never read: the counts are refused first)
    assert lib.topk_combine_fwd(one, 4, one, None, 3, (1 << 25) + 1, 5, 4, 0, one, None) == -1
    assert lib.topk_combine_vjp(one, 4, one, one, one, 4, (1 << 31) - 1, (1 << 31) - 1, 5, 4, 0, one, one, None) == -1


# few places per expert, as in decoding: any length of k and number of columns, one expert with all tokens
@pytest.mark.parametrize("rows,k,n,h,ho", [(1, 1, 1, 4, 32), (1, 2, 8, 4097, 1640), (4, 2, 8, 1003, 2049), (3, 1, 64, 520, 36), (2, 8, 16, 8, 3001),
                                           (8, 1, 8, 2000, 33), (16, 1, 4, 515, 259), (5, 3, 6, 4, 700), (1, 1, 3, 2051, 31), (7, 2, 1024, 64, 64)])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("one", [False, True])
def test_products_of_few_places(gpu, rows, k, n, h, ho, dtype, one):
    import torch
    g = torch.Generator(device="cuda").manual_seed(rows + h)
    dt = getattr(torch, dtype)
    idx = torch.rand((rows, n), generator=g, device="cuda").argsort(dim=1)[:, :k].to(torch.int32).contiguous()
    if one:
        idx[:, 0] = n - 1                                       # (every token, and no other: the rest are empty places)
        idx[:, 1:] = -1
    _, source, offset, _ = gpu.topk_expert_map(idx, n)
    x = torch.randn((rows + 2, h), generator=g, device="cuda").to(dt)
    x[rows:] = float("nan")                                     # (rows that no place names)
    t = torch.randn((rows * k, ho), generator=g, device="cuda").to(dt)
    w = torch.randn((n, ho, h), generator=g, device="cuda").to(dt)
    at = offset.tolist()
    t[at[n]:] = float("inf")
    for transposed in (False, True):
        for shift in (0, 1):
            wd = w.transpose(1, 2).contiguous().transpose(1, 2) if transposed else w
            xd = strided(host(x), dtype, 3, 1) if shift else x
            out = torch.full((rows * k, ho), MARK, device="cuda", dtype=dt)
            gpu.topk_expert_product_fwd(xd, wd, offset, source=source, k=k, out=out)
            dx = torch.full((rows * k, h), MARK, device="cuda", dtype=dt)
            gpu.topk_expert_product_vjp(xd, wd, offset, t, source=source, k=k, dx_out=dx, want_w=False)
            assert (out[at[n]:] == MARK).all() and (dx[at[n]:] == MARK).all()
            for e in range(n):
                if at[e] == at[e + 1]:
                    continue
                part = slice(at[e], at[e + 1])
                xe, te, we = x[(source[part] // k).long()].double(), t[part].double(), w[e].double()
                for have, a, b, terms, name in ((out[part], xe, we.t().contiguous(), h, "out"), (dx[part], te, we, ho, "dx")):
                    want, size = host(a @ b), host(a.abs() @ b.abs())
                    within(host(have), want, (terms + 2) * 2 * U * size + HALF[dtype] * np.abs(want) + TINY[dtype], (name, e))
