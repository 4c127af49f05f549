"""The experts' feed-forward (the gated block, its gradients, 8-bit rows and products) on the GPU against its plain float64 forms
(feed_forward_reference.py), by itself, together, captured, on other streams, and what it refuses.

Two kinds of comparison.  With small whole numbers and max(g, 0) every sum and product is exact, also the slopes in 16 bits (below
256), so that outputs have to EQUAL the exact value rounded once: a place, column or term that is missed, doubled or misplaced
shows.  With real numbers tolerances count roundings, u = 2^-24, HALF[type] half a step of the output's type:
  sums     of K float32 products, every addition off by a step at most: E = (K + 2) 2u sum|a b|.
  act      relative, of the value: silu (2|g| + 8) u: the argument of exp2 is off by |g| 2u, exp2 by 2u, 1 + e by u, the
           reciprocal by 2u, the products by u each.  gelu (2 g^2 + 30) u: exp(-g^2 / 2) off by g^2 u + 2u + 3u, t by 4u and the
           polynomial by 3.2e-7 = 6u, times 2 for the slope of t q(t), products.  gelu_tanh (7 |z| + 8) u, z = 1.6 g (1 + 0.045 g^2),
           whose five roundings count |z| each.  All below 2 |g|^3 u + ..: A(g) below.
  slopes   absolute: twice A (|g| + 1), and their own change with g, at most once the error of g (second derivatives of all
           three are below 1; their slopes below 1.2).
  dx, dW   the errors of the slopes and their rounding to the operands' type, through the sums of absolute values, and E."""
import numpy as np
import pytest

from tests import experts_reference, feed_forward_reference as ref
from tests.test_gpu_experts import HALF, MARK, TINY, U, host, put, rounded, strided, within

pytestmark = pytest.mark.gpu
DTYPES = ("float32", "bfloat16", "float16")


@pytest.fixture(scope="module")
def gpu():
    import torch
    from paper_2302_01425_amd import binding
    assert torch.cuda.is_available()
    binding.load()
    return binding


def act_error(name, g):
    a = np.abs(np.where(np.isfinite(g), g, 0.0))
    z = 1.6 * np.minimum(a, 30.0) * (1.0 + 0.045 * np.minimum(a, 30.0) ** 2)
    return {"silu": 2 * a + 8, "gelu": 2 * np.minimum(a, 15.0) ** 2 + 30, "gelu_tanh": 7 * z + 8, "relu": 0 * a}[name] * U


def case(rows, k, n, h, f, dtype, gather, turned, seed, whole=False, shift=0, pad=0.15):
    """Operands as float64 arrays of values of the type and as tensors, and lists with an expert without places."""
    r = np.random.default_rng(seed)
    idx = np.stack([r.permutation(n)[:k] if n >= k else r.integers(0, n, k) for _ in range(rows)]).astype(np.int32)
    idx[r.random(rows) < pad] = -1
    if n > 2:
        idx[idx == 1] = 0
    slot, source, offset, _ = experts_reference.places(idx, n)
    m = rows if gather else rows * k

    def values(*shape):
        if whole:
            return (r.integers(-1, 2, size=shape) * (r.random(shape) < min(1.0, 12.0 / np.sqrt(h)))).astype(np.float64)
        return rounded(r.normal(size=shape) / (np.sqrt(h) if len(shape) == 3 else 1.0), dtype)

    x, wg, wu, t = values(m, h), values(n, f, h), values(n, f, h), values(rows * k, f)

    def weights(w):
        return put(w.transpose(0, 2, 1), dtype).transpose(1, 2) if turned else put(w, dtype)

    xd = strided(x, dtype, 3, shift) if shift else put(x, dtype)
    td = strided(t, dtype, 1, shift) if shift else put(t, dtype)
    return (x, wg, wu, t), (xd, weights(wg), weights(wu), td), slot, source if gather else None, offset


CASES = [  # rows, k, n, h, f
    (1, 1, 1, 1, 1), (1, 2, 4, 16, 8), (5, 2, 3, 33, 17), (40, 2, 4, 64, 64), (64, 2, 2, 128, 128), (70, 3, 5, 100, 260),
    (300, 1, 2, 136, 72), (130, 2, 1, 31, 129), (9, 4, 40, 256, 128), (260, 2, 3, 72, 264), (700, 2, 3, 328, 520),
    (20, 2, 3, 9, 15), (25, 1, 2, 8, 8), (50, 2, 2, 13, 67), (33, 2, 3, 23, 71), (150, 2, 2, 135, 193), (90, 1, 2, 4, 5),
    (60, 2, 3, 70, 3), (3, 1, 2, 520, 40), (1, 8, 16, 264, 96), (2, 2, 4, 1025, 33), (4, 2, 8, 24, 1030), (35, 1, 1, 3, 2)]


@pytest.mark.parametrize("rows,k,n,h,f", CASES)
@pytest.mark.parametrize("dtype", DTYPES)
def test_whole_numbers(gpu, rows, k, n, h, f, dtype):
    import torch
    for gather in (True, False):
        for turned in (False, True):
            for shift in (0, 1):
                print("case", rows, k, n, h, f, dtype, gather, turned, shift, flush=True)
                (x, wg, wu, t), (xd, gd, ud, td), _, source, offset = case(rows, k, n, h, f, dtype, gather, turned, rows + h, True, shift)
                sd, od, end = None if source is None else put(source, "int32"), put(offset, "int32"), offset[-1]
                out = torch.full((rows * k, f), MARK, device="cuda", dtype=xd.dtype)
                pre = torch.full((rows * k, 2, f), MARK, device="cuda", dtype=xd.dtype)
                got = gpu.topk_expert_gated_fwd(xd, gd, ud, od, source=sd, k=k, act=gpu.TOPK_ACT_RELU, out=out, pre_out=pre)
                assert got[0] is out and got[1] is pre
                want, g, u = ref.gated(x, wg, wu, offset, source, k, "relu")
                assert np.nanmax(np.abs(np.concatenate((g, u, np.zeros((1, f)))))) < 256           # (exact in every type)
                assert (host(out)[end:] == MARK).all() and (host(pre)[end:] == MARK).all(), "a row behind the last place was written"
                assert np.array_equal(host(out)[:end], rounded(want[:end], dtype))
                assert np.array_equal(host(pre)[:end, 0], g[:end]) and np.array_equal(host(pre)[:end, 1], u[:end])
                alone = gpu.topk_expert_gated_fwd(xd, gd, ud, od, source=sd, k=k, act=gpu.TOPK_ACT_RELU)
                assert torch.equal(alone[:end], out[:end])
                dx = torch.full((rows * k, h), MARK, device="cuda", dtype=xd.dtype)
                wants = ref.gated_vjp(x, wg, wu, offset, source, k, "relu", t)
                for kept in (None, pre):
                    dx.fill_(MARK)
                    dxg, dwg, dwu = gpu.topk_expert_gated_vjp(xd, gd, ud, od, td, source=sd, k=k, act=gpu.TOPK_ACT_RELU, pre=kept, dx_out=dx)
                    assert dxg is dx and dwg.stride() == gd.stride() and dwu.stride() == ud.stride()
                    assert (host(dx)[end:] == MARK).all(), "a row behind the last place was written"
                    assert np.array_equal(host(dx)[:end], rounded(wants[0][:end], dtype)), kept is None
                    assert np.array_equal(host(dwg), rounded(wants[1], dtype)) and np.array_equal(host(dwu), rounded(wants[2], dtype))
                only = gpu.topk_expert_gated_vjp(xd, gd, ud, od, td, source=sd, k=k, act=gpu.TOPK_ACT_RELU, want_w=False)
                assert only[1] is None and only[2] is None and torch.equal(only[0][:end], dx[:end])
                only = gpu.topk_expert_gated_vjp(xd, gd, ud, od, td, source=sd, k=k, act=gpu.TOPK_ACT_RELU, want_x=False)
                assert only[0] is None and torch.equal(only[1], dwg) and torch.equal(only[2], dwu)


def whole(shape, g, dtype, share):
    import torch
    v = torch.randint(-1, 2, shape, generator=g, device="cuda", dtype=torch.int8)
    return (v * (torch.rand(shape, generator=g, device="cuda") < share)).to(dtype)


LARGE = [(1500, 2, 24, 1032, 1040), (1500, 2, 24, 1033, 1047), (2100, 1, 6, 2056, 2048), (700, 3, 5, 131, 1411), (3000, 2, 8, 512, 2176),
         (513, 1, 1, 2048, 4100), (6000, 2, 40, 264, 520), (4096, 2, 32, 1024, 768)]


def large_lists(gpu, rows, k, n, g):
    """Experts of very different loads, some tokens padded."""
    import torch
    liked = 1.5 * torch.randn((1, n), generator=g, device="cuda")
    idx = (torch.randn((rows, n), generator=g, device="cuda") + liked).topk(k, dim=1).indices.to(torch.int32).contiguous()
    idx[torch.rand(rows, generator=g, device="cuda") < 0.1] = -1
    _, source, offset, _ = gpu.topk_expert_map(idx, n)
    return source, offset, offset.tolist()


@pytest.mark.parametrize("rows,k,n,h,f", LARGE)
@pytest.mark.parametrize("dtype", DTYPES)
def test_large_whole_numbers(gpu, rows, k, n, h, f, dtype):
    """Sizes of the larger tiles; the sums in float64, expert by expert."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(rows + h)
    dt = getattr(torch, dtype)
    source, offset, at = large_lists(gpu, rows, k, n, g)
    share = min(1.0, 10.0 / h ** 0.5)
    x, t = whole((rows, h), g, dt, share), whole((rows * k, f), g, dt, 0.5)
    for turned in (False, True):
        wg, wu = whole((n, f, h), g, dt, share), whole((n, f, h), g, dt, share)
        if turned:
            wg, wu = (w.transpose(1, 2).contiguous().transpose(1, 2) for w in (wg, wu))
        print("case", rows, k, n, h, f, dtype, turned, flush=True)
        out = torch.full((rows * k, f), MARK, device="cuda", dtype=dt)
        out, pre = gpu.topk_expert_gated_fwd(x, wg, wu, offset, source=source, k=k, act=gpu.TOPK_ACT_RELU, out=out, want_pre=True)
        assert (out[at[n]:] == MARK).all()
        for kept in (None, pre):
            dx = torch.full((rows * k, h), MARK, device="cuda", dtype=dt)
            _, dwg, dwu = gpu.topk_expert_gated_vjp(x, wg, wu, offset, t, source=source, k=k, act=gpu.TOPK_ACT_RELU, pre=kept, dx_out=dx)
            assert (dx[at[n]:] == MARK).all()
            for e in range(n):
                part = slice(at[e], at[e + 1])
                xe, te, ge, ue = x[(source[part] // k).long()].double(), t[part].double(), wg[e].double().contiguous(), wu[e].double().contiguous()
                gs, us = xe @ ge.t().contiguous(), xe @ ue.t().contiguous()
                assert part.start == part.stop or max(gs.abs().max(), us.abs().max()) < 256
                assert torch.equal(out[part], (gs.clamp(min=0) * us).to(dt)), e
                assert torch.equal(pre[part, 0].double(), gs) and torch.equal(pre[part, 1].double(), us), e
                dg, du = te * us * (gs > 0), te * gs.clamp(min=0)
                assert torch.equal(dx[part], (dg @ ge + du @ ue).to(dt)), (e, kept is None)
                assert torch.equal(dwg[e], (dg.t().contiguous() @ xe).to(dt)) and torch.equal(dwu[e], (du.t().contiguous() @ xe).to(dt)), e


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("h,f", [(1032, 1544), (1280, 1536)])
@pytest.mark.parametrize("gather", [True, False])
def test_gradients_of_large_experts(gpu, dtype, h, f, gather):
    """Some thousand places in two experts, a few in the others, none in one; every ninth place without a row of x, whose cotangent is
    infinite; x behind the last place and its cotangent hold NaN."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(h)
    dt = getattr(torch, dtype)
    at = [0, 3000, 3000, 3001, 8000, 8033]
    n, slots, m = 5, 8050, 9000
    share = 10.0 / h ** 0.5
    x, t = whole((m if gather else slots, h), g, dt, share), whole((slots, f), g, dt, 0.5)
    offset = torch.tensor(at, dtype=torch.int32, device="cuda")
    source, gone = None, torch.zeros(slots, dtype=torch.bool, device="cuda")
    if gather:
        source = torch.randint(0, 2 * m, (slots,), generator=g, device="cuda", dtype=torch.int32)
        gone[::9] = True
        source[::18], source[9::18] = -1, 2 * m + 5
        t[gone] = float("inf")
    else:
        x[at[n]:] = float("nan")
    t[at[n]:] = float("nan")
    for turned in (False, True):
        wg, wu = whole((n, f, h), g, dt, share), whole((n, f, h), g, dt, share)
        if turned:
            wg, wu = (w.transpose(1, 2).contiguous().transpose(1, 2) for w in (wg, wu))
        print("case", dtype, h, f, gather, turned, flush=True)
        dx = torch.full((slots, h), MARK, device="cuda", dtype=dt)
        _, dwg, dwu = gpu.topk_expert_gated_vjp(x, wg, wu, offset, t, source=source, k=2, act=gpu.TOPK_ACT_RELU, dx_out=dx)
        assert (dx[at[n]:] == MARK).all()
        for e in range(n):
            part = slice(at[e], at[e + 1])
            keep = ~gone[part]
            row = torch.arange(slots, device="cuda")[part] if source is None else torch.where(keep, source[part] // 2, 0).long()
            xe = x[row].double() * keep[:, None]
            te = torch.where(keep[:, None], t[part].double(), 0.0)
            ge, ue = wg[e].double().contiguous(), wu[e].double().contiguous()
            gs, us = xe @ ge.t().contiguous(), xe @ ue.t().contiguous()
            dg, du = te * us * (gs > 0), te * gs.clamp(min=0)
            assert torch.equal(dx[part], (dg @ ge + du @ ue).to(dt)), e
            assert torch.equal(dwg[e], (dg.t().contiguous() @ xe).to(dt)) and torch.equal(dwu[e], (du.t().contiguous() @ xe).to(dt)), e


@pytest.mark.parametrize("rows,k,n,h,f", [(5, 2, 3, 33, 17), (1, 2, 4, 64, 40), (70, 2, 4, 128, 64), (300, 1, 2, 137, 75), (400, 2, 3, 256, 160)])
@pytest.mark.parametrize("name", ref.ACTS)
@pytest.mark.parametrize("dtype", DTYPES)
def test_activations(gpu, rows, k, n, h, f, name, dtype):
    code = ref.ACTS.index(name)
    (x, wg, wu, t), (xd, gd, ud, td), _, source, offset = case(rows, k, n, h, f, dtype, True, False, rows + f, shift=1)
    sd, od, end = put(source, "int32"), put(offset, "int32"), offset[-1]
    xs, there = ref.rows_of(x, offset, source, k)
    (g, sg), (u, su) = ref.sums(xs, wg, offset), ref.sums(xs, wu, offset)
    g, sg, u, su = (a[:end] for a in (g, sg, u, su))
    eg, eu = (h + 2) * 2 * U * sg, (h + 2) * 2 * U * su
    out, pre = gpu.topk_expert_gated_fwd(xd, gd, ud, od, source=sd, k=k, act=code, want_pre=True)
    half, tiny = HALF[dtype], TINY[dtype]
    within(host(pre)[:end, 0], g, eg + half * np.abs(g) + tiny, "g")
    within(host(pre)[:end, 1], u, eu + half * np.abs(u) + tiny, "u")
    kept = host(pre)
    for which in ("again", "kept"):
        if which == "kept":
            g, u, eg, eu = kept[:end, 0], kept[:end, 1], 0 * eg, 0 * eu
        value, slope = ref.act(name, g)
        ev = 1.2 * eg + act_error(name, g) * np.abs(value) + 2.0 ** -126 * (1 + np.abs(g))
        es = eg + 2 * act_error(name, g) * (np.abs(g) + 1) + 8 * U
        if name == "relu":
            es = np.where(np.abs(g) <= eg, 1.0, 0.0)
        if which == "again":
            want = value * u
            within(host(out)[:end], want, ev * np.abs(u) + np.abs(value) * eu + ev * eu + (half + 2 * U) * np.abs(want) + tiny, "out")
        tt = t[:end]
        dg, du = tt * u * slope, tt * value
        edg = np.abs(tt) * (eu * np.abs(slope) + (np.abs(u) + eu) * es) + (half + 4 * U) * np.abs(dg) + tiny
        edu = np.abs(tt) * ev + (half + 4 * U) * np.abs(du) + tiny
        pad = np.full((rows * k - end, f), np.nan)
        full = [np.concatenate((a, pad)) for a in (dg, du, edg, edu, np.abs(dg) + edg, np.abs(du) + edu)]
        wants = ref.back(full[0], full[1], xs, wg, wu, offset)
        errors = ref.back(full[2], full[3], np.abs(xs), np.abs(wg), np.abs(wu), offset)
        sizes = ref.back(full[4], full[5], np.abs(xs), np.abs(wg), np.abs(wu), offset)
        got = gpu.topk_expert_gated_vjp(xd, gd, ud, od, td, source=sd, k=k, act=code, pre=None if which == "again" else pre)
        terms = (2 * f, max(1, int(np.diff(offset).max())), max(1, int(np.diff(offset).max())))
        for have, want, error, size, count, what in zip(got, wants, errors, sizes, terms, ("dx", "dw_gate", "dw_up")):
            have = host(have)
            if what == "dx":
                have, want, error, size = have[:end], want[:end], error[:end], size[:end]
            within(have, want, error + (count + 2) * 2 * U * size + half * np.abs(want) + tiny, (which, what))


@pytest.mark.parametrize("name", ref.ACTS)
@pytest.mark.parametrize("dtype", DTYPES)
def test_activations_everywhere(gpu, name, dtype):
    """One weight of 1 each: g and u are x itself, from the smallest to the largest, infinities and NaN among them."""
    big = {"float32": 1e38, "bfloat16": 1e38, "float16": 6e4}[dtype]
    x = np.concatenate((np.linspace(-30, 30, 2001), np.linspace(-1e-3, 1e-3, 64), [0.0, -0.0, 100.0, -100.0, 1e4, -1e4, big, -big, np.inf, np.nan]))
    x = rounded(x, dtype).reshape(-1, 1)
    one, zero = np.ones((1, 1, 1)), np.zeros((1, 1))
    off = put(np.array([0, len(x)], np.int32), "int32")
    code = ref.ACTS.index(name)
    # u = 1 with the gate's sum given: the backward pass from kept sums gives du = t act(g), dg = t act'(g) alone, through W = 1
    import torch
    pre = torch.stack((put(x, dtype), put(np.ones_like(x), dtype)), dim=1).contiguous()
    t = put(np.ones_like(x), dtype)
    value, slope = ref.act(name, np.where(np.abs(x) > 1e3, np.sign(x) * 1e3, x))
    value = np.where(x > 1e3, x, value)
    with np.errstate(invalid="ignore"):
        ev = act_error(name, x) * np.abs(value) + 2.0 ** -126 * (1 + np.abs(np.clip(x, -1e3, 1e3)))
    es = 2 * act_error(name, np.clip(x, -30, 30)) * (np.abs(np.clip(x, -30, 30)) + 1) + 8 * U
    ok = np.isfinite(x)
    gate = gpu.topk_expert_gated_vjp(put(x, dtype), put(one, dtype), put(zero[None], dtype), off, t, act=code, pre=pre, want_w=False)[0]
    up = gpu.topk_expert_gated_vjp(put(x, dtype), put(zero[None], dtype), put(one, dtype), off, t, act=code, pre=pre, want_w=False)[0]
    # (0 * infinity in the half that is left out is NaN, as in the formula: finite rows only)
    within(host(gate)[ok], slope[ok], (es + (2 * HALF[dtype] + 4 * U) * np.abs(slope) + TINY[dtype])[ok], "slope")
    within(host(up)[ok], value[ok], (ev + (2 * HALF[dtype] + 4 * U) * np.abs(value) + TINY[dtype])[ok], "value")
    y = host(gpu.topk_expert_gated_fwd(put(x, dtype), put(one, dtype), put(one, dtype), off, act=code))
    small = np.abs(x) < 1e2
    want = value * x
    within(y[small], want[small], (ev * np.abs(x) + (HALF[dtype] + 4 * U) * np.abs(want) + TINY[dtype])[small], "out")
    assert np.isnan(y[np.isnan(x)]).all()
    assert (y[np.isposinf(x)] == np.inf).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("h,f", [(16, 8), (24, 40), (33, 7)])
def test_places_without_a_row(gpu, dtype, h, f):
    """Sources out of range: zeros in every output, nothing in dW, whatever weights, cotangents and kept sums hold."""
    import torch
    r = np.random.default_rng(4)
    x = rounded(r.integers(-1, 2, size=(6, h)), dtype)
    wg, wu = (rounded(r.integers(-1, 2, size=(2, f, h)), dtype) for _ in range(2))
    t = rounded(r.integers(-1, 2, size=(8, f)), dtype)
    source, offset = np.array([0, 3, -5, 2 ** 31 - 1, 12, 11, 7, 4], np.int32), np.array([0, 5, 8], np.int32)
    out_of = [2, 3, 4]
    t[out_of] = np.inf
    lists = (put(offset, "int32"), put(source, "int32"))
    out, pre = gpu.topk_expert_gated_fwd(put(x, dtype), put(wg, dtype), put(wu, dtype), lists[0], lists[1], 2, gpu.TOPK_ACT_RELU, True)
    want, g, u = ref.gated(x, wg, wu, offset, source, 2, "relu")
    assert np.array_equal(host(out), rounded(want, dtype)) and (host(out)[out_of] == 0).all() and (host(pre)[out_of] == 0).all()
    wants = ref.gated_vjp(x, wg, wu, offset, source, 2, "relu", t)
    bad = pre.clone()
    bad[out_of] = float("nan")
    for kept in (None, pre, bad):
        got = gpu.topk_expert_gated_vjp(put(x, dtype), put(wg, dtype), put(wu, dtype), lists[0], put(t, dtype), lists[1], 2,
                                        gpu.TOPK_ACT_RELU, kept)
        for a, b in zip(got, wants):
            assert np.array_equal(host(a), rounded(b, dtype))
    # infinite weights of the expert: its place without a row stays zero
    wi = wg.copy()
    wi[0] = np.inf
    for args in ((wi, wu), (wg, wi), (wi, wi)):
        y, p = gpu.topk_expert_gated_fwd(put(x, dtype), *(put(w, dtype) for w in args), lists[0], lists[1], 2, gpu.TOPK_ACT_SILU, True)
        assert (host(y)[out_of] == 0).all() and (host(p)[out_of] == 0).all()
        dx = gpu.topk_expert_gated_vjp(put(x, dtype), *(put(w, dtype) for w in args), lists[0], put(t, dtype), lists[1], 2, want_w=False)[0]
        assert (host(dx)[out_of] == 0).all()
    # no rows at all
    empty = gpu.topk_expert_gated_fwd(torch.empty((0, h), device="cuda", dtype=pre.dtype), put(wg, dtype), put(wu, dtype), *lists, 2)
    assert (host(empty) == 0).all()
    # offsets outside the places are cut off, unordered ones are read as they are: nothing out of range is touched
    for cut in ([-7, 5, 100], [0, 5, 3], [2 ** 31 - 1, 0, 8], [-2 ** 31, -2 ** 31, 2 ** 31 - 1]):
        o = put(np.array(cut, np.int32), "int32")
        gpu.topk_expert_gated_fwd(put(x, dtype), put(wg, dtype), put(wu, dtype), o, lists[1], 2)
        gpu.topk_expert_gated_vjp(put(x, dtype), put(wg, dtype), put(wu, dtype), o, put(t, dtype), lists[1], 2)
        gpu.topk_expert_gated_vjp(put(x, dtype), put(wg, dtype), put(wu, dtype), o, put(t, dtype), lists[1], 2, pre=pre)
    torch.cuda.synchronize()


# every kernel that takes rows of 16 bits: few, thin (of half the columns, and of all), small, middle and large tiles
KERNELS = [(6, 2, 3, 64, 40), (120, 2, 3, 512, 512), (120, 2, 3, 512, 1024), (300, 2, 2, 129, 1141), (2600, 2, 4, 264, 520), (12000, 2, 8, 1024, 768)]


@pytest.mark.parametrize("rows,k,n,h,f", KERNELS)
@pytest.mark.parametrize("name", ref.ACTS)
@pytest.mark.parametrize("dtype", DTYPES)
def test_nan_stays_in_its_row(gpu, rows, k, n, h, f, name, dtype):
    """A NaN in a token makes its places NaN in every output, and nothing else (dW: its experts)."""
    import torch
    code = ref.ACTS.index(name)
    g = torch.Generator(device="cuda").manual_seed(3)
    dt = getattr(torch, dtype)
    x = torch.randn((rows, h), generator=g, device="cuda").to(dt)
    wg, wu = ((torch.randn((n, f, h), generator=g, device="cuda") / h ** 0.5).to(dt) for _ in range(2))
    idx = torch.rand((rows, n), generator=g, device="cuda").argsort(dim=1)[:, :k].int().contiguous()
    idx[rows // 2, 0], idx[rows // 2, 1:] = 0, -1                   # the token that is NaN: one place, of the first expert
    x[rows // 2, h - 1] = float("nan")
    slot, source, offset, _ = gpu.topk_expert_map(idx, n)
    t = torch.randn((rows * k, f), generator=g, device="cuda").to(dt)
    last, mine = int(offset[n]), int(slot[rows // 2, 0])
    out, pre = gpu.topk_expert_gated_fwd(x, wg, wu, offset, source, k, code, True)
    for kept in (None, pre):
        dx, dwg, dwu = gpu.topk_expert_gated_vjp(x, wg, wu, offset, t, source, k, code, kept)
        for a in (out, pre.flatten(1), dx):
            bad = torch.isnan(a[:last])
            assert bad[mine].all() and int(bad.sum()) == a.shape[1]
        assert torch.isnan(dwg[0]).all() and torch.isnan(dwu[0]).all() and not torch.isnan(dwg[1:]).any() and not torch.isnan(dwu[1:]).any()


@pytest.mark.parametrize("rows,k,n,h,f", KERNELS + [(6000, 2, 4, 1032, 1544)])
@pytest.mark.parametrize("dtype", DTYPES)
def test_whatever_lies_behind(gpu, rows, k, n, h, f, dtype):
    """Scratch that holds NaN, tokens that no place has, and places behind the last, NaN too: outputs as without them, what lies
    behind the last place as it was."""
    import ctypes
    import torch
    g = torch.Generator(device="cuda").manual_seed(9)
    dt = getattr(torch, dtype)
    x = torch.randn((rows, h), generator=g, device="cuda").to(dt)
    wg, wu = ((torch.randn((n, f, h), generator=g, device="cuda") / h ** 0.5).to(dt) for _ in range(2))
    idx = torch.rand((rows, n), generator=g, device="cuda").argsort(dim=1)[:, :k].int().contiguous()
    idx[::7] = -1
    _, source, offset, _ = gpu.topk_expert_map(idx, n)
    last, slots = int(offset[n]), rows * k
    t = torch.randn((slots, f), generator=g, device="cuda").to(dt)
    want = gpu.topk_expert_gated_vjp(x, wg, wu, offset, t, source, k)
    y, pre = gpu.topk_expert_gated_fwd(x, wg, wu, offset, source, k, want_pre=True)
    x[::7], t[last:], source[last:] = float("nan"), float("nan"), 7 * k
    lib, p = gpu.load(), lambda v: None if v is None else v.data_ptr()
    need = lib.topk_expert_gated_vjp_bytes(slots, f, DTYPES.index(dtype))
    kept_want = gpu.topk_expert_gated_vjp(x, wg, wu, offset, t, source, k, pre=pre)
    pre[last:] = float("nan")
    for kept, wanted in ((None, want), (pre, kept_want)):
        scratch = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
        dx, dwg, dwu = torch.full((slots, h), 5.0, device="cuda", dtype=dt), torch.empty_like(wg), torch.empty_like(wu)
        rc = lib.topk_expert_gated_vjp(p(x), h, rows, p(wg), p(wu), f * h, h, 1, p(offset), p(source), k, slots, n, h, f,
                                       DTYPES.index(dtype), 0, p(kept), p(t), f, p(dx), p(dwg), p(dwu), p(scratch), need,
                                       ctypes.c_void_p(torch.cuda.current_stream().cuda_stream))
        assert rc == 0
        assert torch.equal(dx[:last], wanted[0][:last]) and torch.equal(dwg, wanted[1]) and torch.equal(dwu, wanted[2])
        assert (dx[last:] == 5.0).all()
    out, sums = torch.full_like(y, 5.0), torch.full_like(pre, 5.0)
    gpu.topk_expert_gated_fwd(x, wg, wu, offset, source, k, out=out, pre_out=sums)
    assert torch.equal(out[:last], y[:last]) and torch.equal(sums[:last], pre[:last]) and (out[last:] == 5.0).all() and (sums[last:] == 5.0).all()


# W with one row per k (turned weights, dx): widths at which its tiles of 32, 64 and 128 columns end, overlap or do not fit, depths at
# which a step of 8 or 16, times four wavefronts, and the parts of it end
@pytest.mark.parametrize("h,f", [(31, 33), (32, 31), (64, 32), (65, 64), (127, 65), (129, 127), (4, 128), (9, 130), (263, 96), (520, 257)])
@pytest.mark.parametrize("rows", [1, 33, 100])
@pytest.mark.parametrize("dtype", DTYPES)
def test_one_row_per_k(gpu, rows, h, f, dtype):
    (x, wg, wu, t), (xd, gd, ud, td), k, source, offset = case(rows, 2, 3, h, f, dtype, True, True, rows + h + f, True)
    sd, od, end = put(source, "int32"), put(offset, "int32"), offset[-1]
    out, pre = gpu.topk_expert_gated_fwd(xd, gd, ud, od, sd, 2, gpu.TOPK_ACT_RELU, True)
    want, g, u = ref.gated(x, wg, wu, offset, source, 2, "relu")
    assert np.nanmax(np.abs(np.concatenate((g, u, np.zeros((1, f)))))) < 256
    assert np.array_equal(host(out)[:end], rounded(want[:end], dtype)) and np.array_equal(host(pre)[:end, 0], g[:end])
    wants = ref.gated_vjp(x, wg, wu, offset, source, 2, "relu", t)
    for weights in ((gd, ud), (gd.contiguous(), ud.contiguous())):
        for kept in (None, pre):
            got = gpu.topk_expert_gated_vjp(xd, *weights, od, td, sd, 2, gpu.TOPK_ACT_RELU, kept)
            assert np.array_equal(host(got[0])[:end], rounded(wants[0][:end], dtype))
            assert np.array_equal(host(got[1]), rounded(wants[1], dtype)) and np.array_equal(host(got[2]), rounded(wants[2], dtype))


def test_no_places(gpu):
    import torch
    w, x, off = torch.randn((3, 5, 4), device="cuda"), torch.empty((0, 4), device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
    out, pre = gpu.topk_expert_gated_fwd(x, w, w, off, want_pre=True)
    assert out.shape == (0, 5) and pre.shape == (0, 2, 5)
    dx, dg, du = gpu.topk_expert_gated_vjp(x, w, w, off, torch.empty((0, 5), device="cuda"))
    assert dx.shape == (0, 4) and (dg == 0).all() and (du == 0).all()
    # places that no expert has: all rows behind the last place, and zeros for the weights
    x = torch.randn((6, 4), device="cuda")
    out = torch.full((6, 5), MARK, device="cuda")
    gpu.topk_expert_gated_fwd(x, w, w, off, out=out)
    assert (out == MARK).all()
    dx, dg, du = gpu.topk_expert_gated_vjp(x, w, w, off, torch.randn((6, 5), device="cuda"), dx_out=torch.full((6, 4), MARK, device="cuda"))
    assert (dx == MARK).all() and (dg == 0).all() and (du == 0).all()
    q, s = gpu.topk_quantise_rows(torch.empty((0, 7), device="cuda"))
    assert q.shape == (0, 7) and s.shape == (0,)
    wq, ws = w.to(torch.int8), torch.ones((3, 5), device="cuda")
    assert gpu.topk_expert_product_i8_fwd(torch.empty((0, 4), dtype=torch.int8, device="cuda"), s, wq, ws, off).shape == (0, 5)


def test_two_parts_of_one_array(gpu):
    """Gate and up as halves of one [n, 2 f, h] array, and interleaved rows of one."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(3)
    w = torch.randn((3, 128, 72), generator=g, device="cuda", dtype=torch.bfloat16)
    x = torch.randn((50, 72), generator=g, device="cuda", dtype=torch.bfloat16)
    off = torch.tensor([0, 20, 20, 50], dtype=torch.int32, device="cuda")
    for a, b in ((w[:, :64], w[:, 64:]), (w[:, 64:], w[:, :64]), (w[:, ::2], w[:, 1::2])):
        out = gpu.topk_expert_gated_fwd(x, a, b, off)
        assert torch.equal(out, gpu.topk_expert_gated_fwd(x, a.contiguous(), b.contiguous(), off))
    # one array twice: max(g, 0)^2, g as the plain product rounds it (half a step), with the errors of both sums
    same = gpu.topk_expert_gated_fwd(x, w, w, off, act=gpu.TOPK_ACT_RELU)
    p = host(gpu.topk_expert_product_fwd(x, w, off)).clip(min=0)
    size = 1.01 * host(gpu.topk_expert_product_fwd(x.abs(), w.abs(), off))
    e = 2 * (72 + 2) * 2 * U * size + 2.0 ** -8 * p
    within(host(same), p * p, 2 * p * e + e * e + 2.0 ** -8 * (p + e) ** 2, "square")


# ---- 8 bits -----------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("m,h", [(1, 1), (3, 2), (5, 7), (4, 8), (70, 9), (33, 64), (8, 257), (6, 1001), (3, 2048), (5, 4096), (2, 4099),
                                 (3, 8200), (2, 16384), (2, 20003), (1, 70001), (513, 40)])
@pytest.mark.parametrize("dtype", DTYPES)
def test_quantise(gpu, m, h, dtype):
    import torch
    r = np.random.default_rng(m + h)
    for shift in (0, 1):
        x = r.normal(size=(m, h)) * np.exp(r.normal(size=(m, 1)))
        if m > 4:
            x[0] = 0.0
            x[1] = np.round(x[1] * 8) / 8
            x[2] = np.clip(np.round(x[2] * 40) * 0.5, -126.5, 126.5)
            x[2, -1] = 127.0                                # q = x: many halves
            x[3, h // 2] = np.nan
            x[4, 0] = -np.inf
        x = rounded(x, dtype)
        xd = strided(x, dtype, 3, 1) if shift else put(x, dtype)
        q = torch.full((m, h), 77, dtype=torch.int8, device="cuda")
        s = torch.full((m,), MARK, device="cuda")
        got = gpu.topk_quantise_rows(xd, q_out=q, scale_out=s)
        assert got[0] is q and got[1] is s
        wq, ws = ref.quantise(x)
        print("case", m, h, dtype, shift, flush=True)
        assert np.array_equal(host(q), wq)
        assert np.array_equal(host(s).astype(np.float32), ws.astype(np.float32), equal_nan=True)


@pytest.mark.parametrize("h", [64, 513, 2048])
@pytest.mark.parametrize("dtype", DTYPES)
def test_quantise_beside_halves(gpu, h, dtype):
    """Quotients at a half and a few steps of the type beside it: 127 x and (H + 1/2) a are exact in float64, and compared."""
    import torch
    r = np.random.default_rng(h)
    m = 300
    low, high = (-90, 100) if dtype != "float16" else (-8, 12)
    a = rounded(np.ldexp(1.0 + r.random(m), r.integers(low, high, m)), dtype)
    half = r.integers(0, 127, (m, h)) + 0.5
    steps = r.integers(-3, 4, (m, h))
    x = rounded(half * a[:, None] / 127.0, dtype)
    x = np.clip(rounded(x * (1.0 + steps * 2 * HALF[dtype]), dtype), 0.0, a[:, None]) * r.choice([-1.0, 1.0], (m, h))
    x[:, h // 2] = a
    if dtype != "float32":
        x[:, ::5] = x[:, ::5] / np.abs(x[:, ::5]) * a[:, None] / 2          # quotient 63.5
    assert np.array_equal(x, rounded(x, dtype))
    n = np.floor(127.0 * np.abs(x) / a[:, None] + 0.25)                     # the half beside which it lies, or none near
    whole = np.rint(127.0 * np.abs(x) / a[:, None])
    gap = 127.0 * np.abs(x) - (n + 0.5) * a[:, None]
    near = np.abs(127.0 * np.abs(x) / a[:, None] - (n + 0.5)) < 0.1
    want = np.where(near, np.where(gap > 0, n + 1, np.where(gap < 0, n, 2 * np.ceil(n / 2))), whole) * np.sign(x)
    q, scale = gpu.topk_quantise_rows(put(x, dtype))
    assert np.array_equal(host(q), want)
    assert np.array_equal(host(scale).astype(np.float32), (a.astype(np.float32) / np.float32(127.0)))


def test_quantise_at_the_ends_of_float32(gpu):
    tiny = np.float64(2.0) ** -149
    x = np.array([[tiny, -tiny, 0, 3 * tiny], [2.0 ** -126, 2.0 ** -127, -2.0 ** -130, 0], [3.4e38, -3.4e38, 1e38, 1.0],
                  [2.0 ** -118, 2.0 ** -119, 2.0 ** -125, -2.0 ** -118], [1e-36, 3e-37, -1e-38, 5e-39], [1.0, 2.0 ** -9, 1 / 254, -1.0]])
    x = x.astype(np.float32).astype(np.float64)
    q, s = gpu.topk_quantise_rows(put(x))
    wq, ws = ref.quantise(x)
    assert np.array_equal(host(q), wq)
    assert np.array_equal(host(s).astype(np.float32), ws.astype(np.float32))


EIGHTS = CASES + [(200, 2, 3, 1001, 77), (260, 1, 1, 513, 300), (17, 1, 2, 15, 33), (12, 2, 3, 17, 16)]


@pytest.mark.parametrize("rows,k,n,h,f", EIGHTS)
@pytest.mark.parametrize("dtype", DTYPES)
def test_products_of_8_bits(gpu, rows, k, n, h, f, dtype):
    """Scales that are powers of two: the exact sums, rounded once.  Any scales: three roundings more."""
    import torch
    dt = getattr(torch, dtype)
    r = np.random.default_rng(rows + h + f)
    for gather in (True, False):
        for shift in (0, 1):
            _, _, _, source, offset = case(rows, k, n, 1, 1, "float32", gather, False, rows + h)
            m = rows if gather else rows * k
            q, wg, wu = (r.integers(-128, 128, size=s) for s in ((m, h), (n, f, h), (n, f, h)))
            if shift:
                buf = torch.full((m * (h + 3) + 9,), 77, dtype=torch.int8, device="cuda")
                qd = buf[1:1 + m * (h + 3)].view(m, h + 3)[:, :h]
                qd.copy_(put(q, "int8"))
                gd, ud = (torch.full((n, f + 1, h + 5), 77, dtype=torch.int8, device="cuda")[:, :f, 2:h + 2] for _ in range(2))
                gd.copy_(put(wg, "int8")), ud.copy_(put(wu, "int8"))
            else:
                qd, gd, ud = put(q, "int8"), put(wg, "int8"), put(wu, "int8")
            sd, od, end = None if source is None else put(source, "int32"), put(offset, "int32"), offset[-1]
            xs, _ = ref.rows_of(q.astype(np.float64), offset, source, k)
            for exact in (True, False):
                print("case", rows, k, n, h, f, dtype, gather, shift, exact, flush=True)
                scales = [(2.0 ** r.integers(-3, 2, size=s) if exact else r.random(s) + 0.1) * 2.0 ** -6
                          for s in ((m,), (n, f), (n, f))]
                scales = [rounded(s, "float32") for s in scales]
                xsc = ref.rows_of(scales[0][:, None], offset, source, k)[0]
                wants = []
                for w, ws in ((wg, scales[1]), (wu, scales[2])):
                    v = ref.sums(xs, w.astype(np.float64), offset)[0]
                    for e in range(n):
                        v[offset[e]:offset[e + 1]] *= xsc[offset[e]:offset[e + 1]] * ws[e]
                    wants.append(v)
                out = torch.full((rows * k, f), MARK, device="cuda", dtype=dt)
                assert gpu.topk_expert_product_i8_fwd(qd, put(scales[0]), gd, put(scales[1]), od, sd, k, dt, out=out) is out
                assert (host(out)[end:] == MARK).all()
                want = wants[0][:end]
                if exact:
                    assert np.array_equal(host(out)[:end], rounded(want, dtype))
                else:
                    within(host(out)[:end], want, (HALF[dtype] + 4 * U) * np.abs(want) + TINY[dtype], "out")
                for code in ((3,) if exact else (0, 1, 2)):
                    y = torch.full((rows * k, f), MARK, device="cuda", dtype=dt)
                    got = gpu.topk_expert_gated_i8_fwd(qd, put(scales[0]), gd, put(scales[1]), ud, put(scales[2]), od, sd, k, code, dt, out=y)
                    assert got is y and (host(y)[end:] == MARK).all()
                    g, u = wants[0][:end], wants[1][:end]
                    value = ref.act(ref.ACTS[code], g)[0]
                    if exact and dtype == "float32":       # (both sums exact, and their product rounded once)
                        assert np.array_equal(host(y)[:end], rounded(value * u, dtype))
                    elif exact:
                        # the product of two exact numbers of float32, rounded to float32 (u of it) and then to the type, or to the
                        # type at once where one instruction multiplies and converts: half a step of what is off by u at most
                        bound = (HALF[dtype] * (1 + U) + U) * np.abs(value * u) + TINY[dtype]
                        over = {"float16": 65520.0, "bfloat16": 3.4e38}[dtype]
                        fits = np.abs(value * u) < over * (1 - 2 * U)
                        within(host(y)[:end][fits], (value * u)[fits], bound[fits], "gated")
                        assert np.isinf(host(y)[:end][np.abs(value * u) >= over * (1 + 2 * U)]).all()
                    else:
                        ev = 1.2 * 4 * U * np.abs(g) + act_error(ref.ACTS[code], g) * np.abs(value) + 2.0 ** -126 * (1 + np.abs(g))
                        bound = ev * np.abs(u) * (1 + 4 * U) + (HALF[dtype] + 8 * U) * np.abs(value * u) + TINY[dtype]
                        within(host(y)[:end], value * u, bound, "gated")


@pytest.mark.parametrize("rows,k,n,h,f", LARGE + [(2000, 2, 4, 4096, 2048)])
def test_large_products_of_8_bits(gpu, rows, k, n, h, f):
    import torch
    g = torch.Generator(device="cuda").manual_seed(rows + h)
    source, offset, at = large_lists(gpu, rows, k, n, g)
    q, wg, wu = (torch.randint(-127, 128, s, generator=g, device="cuda", dtype=torch.int8) for s in ((rows, h), (n, f, h), (n, f, h)))
    ones, each = torch.full((rows,), 0.25, device="cuda"), torch.full((n, f), 2.0 ** -9, device="cuda")
    each[:, ::3] = 2.0 ** -7
    out = torch.full((rows * k, f), MARK, device="cuda")
    gpu.topk_expert_product_i8_fwd(q, ones, wg, each, offset, source, k, torch.float32, out=out)
    both = torch.full((rows * k, f), MARK, device="cuda")
    gpu.topk_expert_gated_i8_fwd(q, ones, wg, each, wu, each, offset, source, k, gpu.TOPK_ACT_RELU, torch.float32, out=both)
    assert (out[at[n]:] == MARK).all() and (both[at[n]:] == MARK).all()
    for e in range(n):
        part = slice(at[e], at[e + 1])
        xe = q[(source[part] // k).long()].double()
        gs, us = ((xe @ w[e].double().t().contiguous()) * (0.25 * each[e].double()) for w in (wg, wu))
        assert torch.equal(out[part], gs.float()), e          # (whole numbers below 2^53, rounded once; scales powers of two)
        assert torch.equal(both[part], gs.float().clamp(min=0) * us.float()), e


def test_longest_sum_of_8_bits(gpu):
    """131071 products of -128 and -128 just fit 32 bits."""
    import torch
    h = gpu.TOPK_I8_WIDTH_MAX
    q, w = torch.full((3, h), -128, dtype=torch.int8, device="cuda"), torch.full((1, 2, h), -128, dtype=torch.int8, device="cuda")
    off = torch.tensor([0, 3], dtype=torch.int32, device="cuda")
    one, each = torch.ones(3, device="cuda"), torch.ones((1, 2), device="cuda")
    out = gpu.topk_expert_product_i8_fwd(q, one, w, each, off, dtype=torch.float32)
    assert (out == float(np.float32(h * 16384))).all()
    with pytest.raises(gpu.TopkError):
        gpu.topk_expert_product_i8_fwd(torch.zeros((3, h + 1), dtype=torch.int8, device="cuda"), one,
                                       torch.zeros((1, 2, h + 1), dtype=torch.int8, device="cuda"), each, off)


def test_rows_of_nan_in_8_bits(gpu):
    """A token that holds a NaN gives NaN, its neighbours do not, a place without a row gives zeros."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn((6, 40), generator=g, device="cuda")
    x[2, 7] = float("nan")
    q, s = gpu.topk_quantise_rows(x)
    w, ws = gpu.topk_quantise_rows(torch.randn((2 * 24, 40), generator=g, device="cuda"))
    w, ws = w.view(2, 24, 40), ws.view(2, 24)
    off, src = (torch.tensor(v, dtype=torch.int32, device="cuda") for v in ([0, 4, 8], [0, 5, 2, 9, 1, 2, -1, 99]))
    for out in (gpu.topk_expert_product_i8_fwd(q, s, w, ws, off, src, 1), gpu.topk_expert_gated_i8_fwd(q, s, w, ws, w, ws, off, src, 1)):
        assert torch.isnan(out[[2, 5]]).all() and not torch.isnan(out[[0, 1, 3, 4, 6, 7]]).any() and (out[[3, 6, 7]] == 0).all()


# ---- offsets that 32 bits do not hold --------------------------------------------------------------------------------------

def small_whole(shape, dtype, seed, share=1.0):
    """-1, 0 and 1, of which the fraction `share` is not cleared."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    v = torch.empty(shape, dtype=torch.int8, device="cuda").random_(-1, 2, generator=g)
    if share < 1.0:
        v *= torch.empty(shape, dtype=torch.int8, device="cuda").random_(0, int(1 / share), generator=g) == 0
    return v.to(dtype)


def test_many_places_of_wide_rows(gpu):
    """2.3e9 outputs, twice as many kept sums and slopes: the last expert's places as by themselves."""
    import torch
    slots, h, f, relu = 140000, 16, 16384, gpu.TOPK_ACT_RELU
    x, t = small_whole((slots, h), torch.bfloat16, 1), small_whole((slots, f), torch.bfloat16, 2)
    wg, wu = small_whole((3, f, h), torch.bfloat16, 3), small_whole((3, f, h), torch.bfloat16, 4)
    off = torch.tensor([0, 60000, 60000, slots], dtype=torch.int32, device="cuda")
    out, pre = gpu.topk_expert_gated_fwd(x, wg, wu, off, act=relu, want_pre=True)
    last = slice(slots - 3000, slots)
    alone = torch.tensor([0, 3000], dtype=torch.int32, device="cuda")
    want, sums = gpu.topk_expert_gated_fwd(x[last], wg[2:], wu[2:], alone, act=relu, want_pre=True)
    assert torch.equal(out[last], want) and torch.equal(pre[last], sums)
    del out
    wants = gpu.topk_expert_gated_vjp(x[last], wg[2:], wu[2:], alone, t[last], act=relu)
    for kept in (None, pre):
        dx, dwg, dwu = gpu.topk_expert_gated_vjp(x, wg, wu, off, t, act=relu, pre=kept)
        assert torch.equal(dx[last], wants[0])
        # sums of whole numbers below 2^24, in any order
        g, u = (x[60000:].float() @ w[2].float().t().contiguous() for w in (wg, wu))
        tf = t[60000:].float()
        assert torch.equal(dwu[2], ((tf * g.clamp(min=0)).t().contiguous() @ x[60000:].float()).bfloat16())
        assert torch.equal(dwg[2], ((tf * u * (g > 0)).t().contiguous() @ x[60000:].float()).bfloat16())
        assert (dwg[1] == 0).all() and (dwu[1] == 0).all()
        del g, u, tf


@pytest.mark.parametrize("places", [5, 100, 700])
def test_rows_and_weights_far_apart(gpu, places):
    """Tokens of 2.2e9 values, weights of 2.7e9: rows at the end, by experts at the end, as by themselves; 16 and 8 bits."""
    import torch
    m, h, n, f, relu = 270000, 8192, 40, 8192, gpu.TOPK_ACT_RELU
    g = torch.Generator(device="cuda").manual_seed(places)
    rows = m - 1 - torch.randperm(2000, generator=g, device="cuda")[:places]
    source = (2 * rows + 1).int()
    off = torch.zeros(n + 1, dtype=torch.int32, device="cuda")
    off[n - 1], off[n] = places // 3, places
    alone = off[n - 2:].contiguous()
    t = small_whole((places, f), torch.bfloat16, 3)
    for dtype in (torch.bfloat16, torch.int8):
        x = torch.zeros((m, h), dtype=dtype, device="cuda")
        x[-2000:] = small_whole((2000, h), dtype, 1, 0.01)
        wg, wu = (torch.zeros((n, f, h), dtype=dtype, device="cuda") for _ in range(2))
        wg[n - 2:], wu[n - 2:] = small_whole((2, f, h), dtype, 4), small_whole((2, f, h), dtype, 5)
        if dtype == torch.int8:
            one, each = torch.ones(m, device="cuda"), torch.ones((n, f), device="cuda")
            got = gpu.topk_expert_gated_i8_fwd(x, one, wg, each, wu, each, off, source, 2, relu, torch.float32)
            want = gpu.topk_expert_gated_i8_fwd(x[rows], one[:places], wg[n - 2:], each[:2], wu[n - 2:], each[:2], alone, None, 1, relu,
                                                torch.float32)
            assert torch.equal(got, want) and (want != 0).any()
            got = gpu.topk_expert_product_i8_fwd(x, one, wg, each, off, source, 2, torch.float32)
            assert torch.equal(got, gpu.topk_expert_product_i8_fwd(x[rows], one[:places], wg[n - 2:], each[:2], alone, dtype=torch.float32))
        else:
            got = gpu.topk_expert_gated_fwd(x, wg, wu, off, source, 2, relu)
            want = gpu.topk_expert_gated_fwd(x[rows], wg[n - 2:], wu[n - 2:], alone, None, 1, relu)
            assert torch.equal(got, want) and (want != 0).any()
            back = gpu.topk_expert_gated_vjp(x, wg, wu, off, t, source, 2, relu)
            wants = gpu.topk_expert_gated_vjp(x[rows], wg[n - 2:], wu[n - 2:], alone, t, None, 1, relu)
            assert torch.equal(back[0], wants[0])
            for a, b in zip(back[1:], wants[1:]):
                assert torch.equal(a[n - 2:], b) and not a[:n - 2].any()


def test_rows_in_8_bits_far_apart(gpu):
    import torch
    x = torch.zeros((270000, 8192), dtype=torch.bfloat16, device="cuda")
    x[-3:] = torch.randn((3, 8192), device="cuda").bfloat16()
    q, scale = gpu.topk_quantise_rows(x)
    q0, s0 = gpu.topk_quantise_rows(x[-3:].clone())
    assert torch.equal(q[-3:], q0) and torch.equal(scale[-3:], s0) and not q[:-3].any() and not scale[:-3].any()


# ---- together, captured, elsewhere -----------------------------------------------------------------------------------------

def layer(gpu, x, logits, wg, wu, wd, k):
    """Forward and backward of a layer: choice, places, gated block, second product, sum per token."""
    idx, val = gpu.topk_route_fwd(logits, k)
    slot, source, offset, _ = gpu.topk_expert_map(idx, logits.shape[1])
    a, pre = gpu.topk_expert_gated_fwd(x, wg, wu, offset, source, k, want_pre=True)
    y = gpu.topk_expert_product_fwd(a, wd, offset)
    out = gpu.topk_combine_fwd(y, slot, val)
    dy, dval = gpu.topk_combine_vjp(y, slot, val, out)                     # the cotangent of |out|^2 / 2
    da, dwd = gpu.topk_expert_product_vjp(a, wd, offset, dy)
    dx, dwg, dwu = gpu.topk_expert_gated_vjp(x, wg, wu, offset, da, source, k, pre=pre)
    return out, gpu.topk_combine_fwd(dx, slot), dwg, dwu, dwd, gpu.topk_route_vjp(logits, idx, dval)


def layer_inputs(dtype, rows=150, n=6, h=72, f=56, seed=0):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = getattr(torch, dtype)
    x = torch.randn((rows, h), generator=g, device="cuda").to(dt)
    w = [(torch.randn(s, generator=g, device="cuda") / s[2] ** 0.5).to(dt) for s in ((n, f, h), (n, f, h), (n, h, f))]
    return x, torch.randn((rows, n), generator=g, device="cuda"), *w


def test_a_layer_against_automatic_gradients(gpu):
    """Float32 against the same formulas in float64 with gradients by torch's own rules."""
    import torch
    x, logits, wg, wu, wd = layer_inputs("float32")
    k = 2
    have = layer(gpu, x, logits, wg, wu, wd, k)
    leaves = [t.double().cpu().requires_grad_() for t in (x, wg, wu, wd, logits)]
    X, G, Uw, D, L = leaves
    idx = L.topk(k, dim=1).indices
    val = torch.softmax(L, 1).gather(1, idx)
    val = val / val.sum(1, keepdim=True)
    out = torch.zeros_like(X)
    for j in range(k):
        rows = []
        for r in range(len(X)):
            e = idx[r, j]
            gate = G[e] @ X[r]
            rows.append(val[r, j] * (D[e] @ (gate / (1 + torch.exp(-gate)) * (Uw[e] @ X[r]))))
        out = out + torch.stack(rows)
    (0.5 * (out * out).sum()).backward()
    wants = (out.detach(), X.grad, G.grad, Uw.grad, D.grad, L.grad)
    for a, b, name in zip(have, wants, ("out", "dx", "dwg", "dwu", "dwd", "dlogits")):
        # every value passes a handful of sums of at most 72 + 56 + 150 terms: (278 + 60) 2u of the size of the largest, as the
        # sums of absolute values here are below 8 times the largest value
        size = 8 * b.abs().max().item()
        assert (a.double().cpu() - b).abs().max().item() <= 338 * 2 * U * size, name


@pytest.mark.parametrize("dtype", DTYPES)
def test_captured_and_replayed(gpu, dtype):
    """Two layers captured into graphs (each with scratch of its own), replayed several times with eager work between."""
    import torch
    sets = [layer_inputs(dtype, seed=s) for s in (1, 2)]
    with torch.cuda.stream(torch.cuda.Stream()):
        for s in sets:
            layer(gpu, *s, 2)
    torch.cuda.synchronize()
    graphs, outs = [], []
    for s in sets:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(layer(gpu, *s, 2))
        graphs.append(g)
    for turn in range(4):
        for s, seed in zip(sets, (10 + turn, 20 + turn)):
            for old, new in zip(s, layer_inputs(dtype, seed=seed)):
                old.copy_(new)
        graphs[turn % 2].replay(), graphs[1 - turn % 2].replay()
        eager = [layer(gpu, *s, 2) for s in sets]
        torch.cuda.synchronize()
        for a, b in zip(outs, eager):
            for i, (p, q) in enumerate(zip(a, b)):
                assert torch.equal(p, q), (turn, i)


def test_captured_in_8_bits(gpu):
    import torch
    x, _, wg, wu, _ = layer_inputs("bfloat16", rows=40)
    n, f, h = wg.shape
    (g8, gs), (u8, us) = (gpu.topk_quantise_rows(w.view(n * f, h)) for w in (wg, wu))
    g8, u8, gs, us = g8.view(n, f, h), u8.view(n, f, h), gs.view(n, f), us.view(n, f)
    off = torch.tensor([0, 5, 9, 9, 20, 33, 40], dtype=torch.int32, device="cuda")

    def step():
        q, s = gpu.topk_quantise_rows(x)
        a = gpu.topk_expert_gated_i8_fwd(q, s, g8, gs, u8, us, off)
        q2, s2 = gpu.topk_quantise_rows(a)
        return gpu.topk_expert_product_i8_fwd(q2, s2, g8.transpose(1, 2).contiguous(), torch.ones((n, h), device="cuda"), off)
    with torch.cuda.stream(torch.cuda.Stream()):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for seed in range(4):
        x.copy_(layer_inputs("bfloat16", rows=40, seed=seed)[0])
        graph.replay()
        eager = step()
        torch.cuda.synchronize()
        assert torch.equal(out, eager)


def test_8_bits_are_near_16(gpu):
    """A served block in 8 bits against the same in float32: every product of q scale is off by half a step of either operand,
    scale (|w| + |x| + 1 / 2 scale ..) / 2 per term."""
    import torch
    x, _, wg, wu, _ = layer_inputs("float32", rows=60)
    n, f, h = wg.shape
    off = torch.tensor([0, 10, 20, 30, 40, 50, 60], dtype=torch.int32, device="cuda")
    q, s = gpu.topk_quantise_rows(x)
    w8, ws = gpu.topk_quantise_rows(wg.view(n * f, h))
    out = gpu.topk_expert_product_i8_fwd(q, s, w8.view(n, f, h), ws.view(n, f), off, dtype=torch.float32).double()
    for e in range(n):
        p = slice(10 * e, 10 * e + 10)
        xe, we, sx, sw = x[p].double(), wg[e].double(), s[p].double(), ws.view(n, f)[e].double()
        want = xe @ we.t().contiguous()
        bound = 0.5 * (sx[:, None] * we.abs().sum(1) + xe.abs().sum(1)[:, None] * sw + 0.5 * h * sx[:, None] * sw) * (1 + 1e-5)
        assert ((out[p] - want).abs() <= bound).all()


def test_other_streams(gpu):
    """Given streams, and the current one: a chain of calls behind a long one sees its results."""
    import torch
    s = layer_inputs("bfloat16", seed=5)
    want = layer(gpu, *s, 2)
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    x, _, wg, wu, _ = s
    late = torch.zeros_like(x)
    off = torch.tensor([0, 20, 40, 60, 80, 100, 150], dtype=torch.int32, device="cuda")
    ref_out, ref_pre = gpu.topk_expert_gated_fwd(x, wg, wu, off, want_pre=True)
    ref_back = gpu.topk_expert_gated_vjp(x, wg, wu, off, ref_out)
    q0, s0 = gpu.topk_quantise_rows(x)
    torch.cuda.synchronize()
    with torch.cuda.stream(st):
        a = torch.randn((3000, 3000), device="cuda")
        for _ in range(10):
            a = a @ a * 1e-3
        late.copy_(x)
    out, pre = gpu.topk_expert_gated_fwd(late, wg, wu, off, want_pre=True, stream=st)
    back = gpu.topk_expert_gated_vjp(late, wg, wu, off, out, pre=None, stream=st)
    q, sc = gpu.topk_quantise_rows(late, stream=st.cuda_stream)
    st.synchronize()
    assert torch.equal(out, ref_out) and torch.equal(pre, ref_pre) and torch.equal(q, q0) and torch.equal(sc, s0)
    assert all(torch.equal(a, b) for a, b in zip(back, ref_back))
    with torch.cuda.stream(st):
        again = layer(gpu, *s, 2)
    st.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(again, want))


def test_calls_that_overlap_in_time(gpu):
    """Two streams at once, scratch of their own: results as one after the other."""
    import torch
    sets = [layer_inputs("bfloat16", rows=3000, h=256, f=320, seed=s) for s in (7, 8)]
    wants = [layer(gpu, *s, 2) for s in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    got = [None, None]
    for _ in range(5):
        for i, (s, st) in enumerate(zip(sets, streams)):
            with torch.cuda.stream(st):
                got[i] = layer(gpu, *s, 2)
    torch.cuda.synchronize()
    for a, b in zip(got, wants):
        assert all(torch.equal(p, q) for p, q in zip(a, b))


def test_refusals(gpu):
    import torch
    f32 = dict(device="cuda")
    x, w, t = torch.randn((8, 16), **f32), torch.randn((2, 4, 16), **f32), torch.randn((8, 4), **f32)
    off = torch.tensor([0, 4, 8], dtype=torch.int32, device="cuda")
    b = gpu

    def no(call):
        with pytest.raises(b.TopkError):
            call()
    no(lambda: b.topk_expert_gated_fwd(x.double(), w.double(), w.double(), off))
    no(lambda: b.topk_expert_gated_fwd(x, w, w.half(), off))
    no(lambda: b.topk_expert_gated_fwd(x, w, w[:, :3], off))
    no(lambda: b.topk_expert_gated_fwd(x, w, w.transpose(1, 2).contiguous().transpose(1, 2), off))        # other strides
    no(lambda: b.topk_expert_gated_fwd(x, w[..., ::2], w[..., ::2], off))
    no(lambda: b.topk_expert_gated_fwd(x, w, w, off[:2]))
    no(lambda: b.topk_expert_gated_fwd(x, w, w, off.long()))
    no(lambda: b.topk_expert_gated_fwd(x, w, w, off, act=4))
    no(lambda: b.topk_expert_gated_fwd(x, w, w, off, source=off[:, None]))
    no(lambda: b.topk_expert_gated_fwd(x, w, w, off, k=0))
    no(lambda: b.topk_expert_gated_fwd(x.t(), w, w, off))
    no(lambda: b.topk_expert_gated_fwd(x, w, w, off, out=t[:4]))
    no(lambda: b.topk_expert_gated_fwd(x, w, w, off, out=w.view(-1)[:32].view(8, 4)))                     # overlaps an input
    both = torch.empty((8, 3, 4), **f32).view(-1)
    no(lambda: b.topk_expert_gated_fwd(x, w, w, off, out=both[:32].view(8, 4), pre_out=both[16:80].view(8, 2, 4)))
    no(lambda: b.topk_expert_gated_vjp(x, w, w, off, t[:7]))
    no(lambda: b.topk_expert_gated_vjp(x, w, w, off, t.half()))
    no(lambda: b.topk_expert_gated_vjp(x, w, w, off, t, pre=torch.empty((8, 8), **f32)))
    no(lambda: b.topk_expert_gated_vjp(x, w, w, off, t, dw_gate_out=w))
    d = torch.empty_like(w)
    no(lambda: b.topk_expert_gated_vjp(x, w, w, off, t, dw_gate_out=d, dw_up_out=d))
    assert b.topk_expert_gated_vjp(x, w, w, off, t, want_x=False, want_w=False) == (None, None, None)
    only = b.topk_expert_gated_vjp(x, w, w, off, t, want_x=False, want_w=False, dw_gate_out=d)
    assert only[0] is None and only[1] is d and only[2] is not None
    q, s = b.topk_quantise_rows(x)
    w8, ws = b.topk_quantise_rows(w.view(8, 16))
    w8, ws = w8.view(2, 4, 16), ws.view(2, 4)
    no(lambda: b.topk_quantise_rows(x.t()))
    no(lambda: b.topk_quantise_rows(x, q_out=torch.empty((8, 15), dtype=torch.int8, device="cuda")))
    no(lambda: b.topk_quantise_rows(x.long()))
    no(lambda: b.topk_expert_product_i8_fwd(x, s, w8, ws, off))
    no(lambda: b.topk_expert_product_i8_fwd(q, s[:7], w8, ws, off))
    no(lambda: b.topk_expert_product_i8_fwd(q, s, w8, ws.t(), off))
    no(lambda: b.topk_expert_product_i8_fwd(q, s, w8.transpose(1, 2).contiguous().transpose(1, 2), ws, off))
    no(lambda: b.topk_expert_product_i8_fwd(q, s, w8, ws, off, dtype=torch.float64))
    no(lambda: b.topk_expert_product_i8_fwd(q, s, w8, ws, off, out=torch.empty((8, 4), **f32)))
    no(lambda: b.topk_expert_gated_i8_fwd(q, s, w8, ws, w8[:, :3], ws, off))
    no(lambda: b.topk_expert_gated_i8_fwd(q, s, w8, ws, w8, ws[:1], off))
    no(lambda: b.topk_expert_gated_i8_fwd(q, s, w8, ws, w8, ws, off, act=7))
    no(lambda: b.topk_expert_gated_i8_fwd(q, s, w8, ws, None, None, off))
    no(lambda: b.topk_expert_gated_i8_fwd(q, s, w8, ws, None, ws, off))
    no(lambda: b.topk_expert_gated_i8_fwd(q, s, w8, ws, w8, None, off))
    no(lambda: b.topk_expert_gated_fwd(x, w, None, off))
    no(lambda: b.topk_expert_gated_vjp(x, w, None, off, t))
    no(lambda: b.topk_expert_gated_vjp(x, w, w, off, None))
