"""The operators behind a router (tests/test_gpu_experts.py) where a call's values or sizes are unusual: scores of groups that
float32 cannot tell apart, infinities and NaN at places that are not there, calls that take more than one launch."""
import numpy as np
import pytest

from tests import experts_reference as ref
from tests.test_gpu_experts import gpu, host, put  # noqa: F401  (gpu: the fixture)

pytestmark = pytest.mark.gpu


# ---- route: scores of groups ----------------------------------------------------------------------------------------------

# Groups whose scores differ by a few roundings of what they are made of: `size` the biases of the two largest, +size and -size
# (top 2: their sum is small, its roundings are not) or +size in every group (top 1).
@pytest.mark.parametrize("n,groups,keep", [(4, 2, 1), (60, 6, 2), (64, 8, 3), (1024, 32, 5)])
@pytest.mark.parametrize("size", [0.5, 10.0, 1e3, 1e5])
@pytest.mark.parametrize("top", [1, 2])
def test_route_of_groups_that_cross_in_float32(gpu, n, groups, keep, size, top):
    rows, width = 200, n // groups
    r = np.random.default_rng(n + top)
    for sigmoid in (False, True):
        bias = np.full((groups, width), -3.0 * size, np.float32)
        bias[:, 0] = size * (1.0 + 0.5 * r.random(groups)) if top == 2 else size
        bias[:, 1] = -bias[:, 0] if top == 2 else 0.0
        if top == 2:
            bias[1::2, :2] = 0.0
        bias = bias.reshape(-1)
        l = r.normal(size=(rows, groups, width)).astype(np.float32)
        l[:, 1:, :2] = l[:, :1, :2]
        l[:, 1:, 0] += (2.0 ** -12 * r.normal(size=(rows, groups - 1)) * r.choice([1.0, 0.1, 0.01], size=(rows, 1))).astype(np.float32)
        l = l.reshape(rows, n)
        # rows whose decision is within the roundings of float64 decide nothing here
        c = ref.scores(l, sigmoid) + bias.astype(np.float64)
        score = np.sort(-np.sort(-c.reshape(rows, groups, width), axis=2)[:, :, :top].sum(axis=2), axis=1)[:, ::-1]
        clear = score[:, keep - 1] - score[:, keep] > 32 * 2.0 ** -53 * (1.0 + 2.0 * size)
        assert clear.sum() > rows // 2
        k = min(2, keep * width)
        want = ref.route(l, k, sigmoid, bias, groups, keep, top)[0]
        print("case", n, groups, keep, size, top, sigmoid, int(clear.sum()), flush=True)
        got = host(gpu.topk_route_fwd(put(l), k, int(sigmoid), bias=put(bias), groups=groups, keep_groups=keep, group_top=top)[0])
        bad = clear & (got != want).any(axis=1)
        assert not bad.any(), (int(bad.sum()), np.flatnonzero(bad)[:4], got[bad][:4], want[bad][:4])


def test_route_of_groups_whose_scores_float32_cannot_hold(gpu):
    """Sums of two biases above the largest float32, infinite ones, and groups that are out."""
    l = np.zeros((3, 8), np.float32)
    l[1] = np.arange(8) / 4
    l[2, 6:] = -np.inf
    for bias in ([3.0e38, 3.0e38, 3.2e38, 3.2e38, 0, 0, 3.1e38, 3.3e38], [3.0e38, -3.0e38, 1.0, 1.0, 0.5, 0.5, 3.3e38, 3.3e38],
                 [np.inf, 0, 1, 1, np.inf, 0.5, 3.0e38, 3.0e38], [-np.inf, -np.inf, -3e38, -3e38, -3.1e38, -3.1e38, 0, np.nan]):
        b = np.array(bias, np.float32)
        for sigmoid in (False, True):
            for keep in (1, 2, 3):
                want = ref.route(l, 2, sigmoid, b, 4, keep, 2)[0]
                got = host(gpu.topk_route_fwd(put(l), 2, int(sigmoid), bias=put(b), groups=4, keep_groups=keep, group_top=2)[0])
                assert np.array_equal(got, want), (bias, sigmoid, keep, got, want)


# ---- products: places whose source is out of range -------------------------------------------------------------------------

def with_holes(rng, places, rows, k):
    """Sources with some out of the rows, and which."""
    import torch
    source = rng.integers(0, max(1, rows * k), size=places).astype(np.int32)
    gone = rng.random(places) < 0.25
    gone[0] = True
    bad = np.array([-1, -2 ** 31, rows * k, 2 ** 31 - 1], np.int32)
    source[gone] = bad[rng.integers(0, 4, size=int(gone.sum()))]
    return source, torch.from_numpy(gone).cuda()


# n experts of `share` places, h -> ho: few places, 256 x 256, 128 x 128, 64 x 64, rows shorter than 16 bytes, no rows of x at all
@pytest.mark.parametrize("n,share,rows,h,ho", [(4, 3, 6, 520, 96), (8, 1024, 300, 64, 1024), (8, 512, 300, 67, 899), (3, 50, 20, 72, 136),
                                               (3, 50, 20, 71, 137), (2, 20, 9, 3, 66), (2, 20, 0, 40, 40)])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("transposed", [False, True])
def test_product_of_absent_rows_is_zero_whatever_w_holds(gpu, n, share, rows, h, ho, dtype, transposed):
    import torch
    k = 2
    source, gone = with_holes(np.random.default_rng(n * h), n * share, rows, k)
    if rows == 0:
        gone[:] = True
    g = torch.Generator(device="cuda").manual_seed(h)
    dt = getattr(torch, dtype)
    x = torch.randn((rows, h), generator=g, device="cuda").to(dt)
    w = torch.randn((n, ho, h), generator=g, device="cuda").to(dt)
    w[:, 1, h // 2], w[:, ho - 1, 0], w[0, :, h - 1] = float("inf"), float("nan"), -float("inf")
    w = w.transpose(1, 2).contiguous().transpose(1, 2) if transposed else w
    offset = torch.arange(0, n * share + 1, share, dtype=torch.int32, device="cuda")
    out = gpu.topk_expert_product_fwd(x, w, offset, source=put(source, "int32"), k=k)
    assert (out[gone] == 0).all()
    if rows:
        there = torch.where(gone, 0, put(source, "int32")).to(torch.int32)
        want = gpu.topk_expert_product_fwd(x, w, offset, source=there, k=k)
        assert torch.equal(out[~gone].nan_to_num(nan=7.0), want[~gone].nan_to_num(nan=7.0))


# n experts of `share` places, h x ho of W: 128 x 256 loaded straight to LDS, 128 x 128, 64 x 64, rows shorter than 16 bytes
@pytest.mark.parametrize("n,share,rows,h,ho", [(32, 70, 300, 1024, 256), (4, 1100, 300, 2048, 1024), (64, 40, 300, 389, 259), (3, 1100, 300, 72, 136),
                                               (3, 50, 20, 71, 137), (2, 20, 9, 3, 66), (2, 20, 0, 40, 40)])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("transposed", [False, True])
def test_weight_gradient_leaves_absent_rows_out(gpu, n, share, rows, h, ho, dtype, transposed):
    """A place whose source is out of range adds nothing to dW, whatever its cotangent holds."""
    import torch
    k = 2
    source, gone = with_holes(np.random.default_rng(n * h), n * share, rows, k)
    if rows == 0:
        gone[:] = True
    g = torch.Generator(device="cuda").manual_seed(h)
    dt = getattr(torch, dtype)
    x = torch.randn((rows, h), generator=g, device="cuda").to(dt)
    w = torch.zeros((n, h, ho), dtype=dt, device="cuda").transpose(1, 2) if transposed else torch.zeros((n, ho, h), dtype=dt, device="cuda")
    t = torch.randn((n * share, ho), generator=g, device="cuda").to(dt)
    offset = torch.arange(0, n * share + 1, share, dtype=torch.int32, device="cuda")
    clean = torch.where(gone[:, None], torch.zeros_like(t), t)
    for value in (float("nan"), float("inf")):
        t[gone] = value
        dw = gpu.topk_expert_product_vjp(x, w, offset, t, source=put(source, "int32"), k=k, want_x=False)[1]
        want = torch.zeros_like(dw)
        if rows:
            there = torch.where(gone, 0, put(source, "int32")).to(torch.int32)
            want = gpu.topk_expert_product_vjp(x, w, offset, clean, source=there, k=k, want_x=False)[1]
        assert torch.isfinite(dw).all() and torch.equal(dw, want)


# ---- calls of several launches ---------------------------------------------------------------------------------------------

# rows of `h` elements, several workgroups long, and more tokens than one launch of such workgroups has
@pytest.mark.parametrize("dtype,rows,h", [("bfloat16", (1 << 23) + 3, 2049), ("float32", 2, 65535 * 1024 + 5), ("bfloat16", 3, 2 * 32768 * 2048 + 9)])
def test_combine_of_long_rows_takes_several_launches(gpu, dtype, rows, h):
    import torch
    g = torch.Generator(device="cuda").manual_seed(rows)
    y = torch.randn((5, h), generator=g, device="cuda").to(getattr(torch, dtype))
    slot = torch.randint(-1, 5, (rows, 1), generator=g, device="cuda", dtype=torch.int32)
    out = gpu.topk_combine_fwd(y, slot)
    step = max(1, (1 << 31) // h)
    for at in range(0, rows, step):
        s = slot[at:at + step, 0]
        want = torch.where(s[:, None] >= 0, y[s.clamp(min=0).long()], torch.zeros((), dtype=y.dtype, device="cuda"))
        assert torch.equal(out[at:at + step], want), at


def test_products_of_more_tiles_than_a_launch_takes(gpu):
    import torch
    slots = (1 << 30) + 70
    x = torch.randn((slots, 1), device="cuda")
    w = torch.tensor([2.0, -0.5], device="cuda").view(2, 1, 1)
    half = slots // 2 + 5
    offset = torch.tensor([0, half, slots], dtype=torch.int32, device="cuda")
    out = gpu.topk_expert_product_fwd(x, w, offset)
    assert torch.equal(out[:half], 2.0 * x[:half]) and torch.equal(out[half:], -0.5 * x[half:])
    del out, x
    n, h = 1024, (1 << 20) + 9
    x, t = torch.randn((5, h), device="cuda"), torch.randn((5, 1), device="cuda")
    offset = torch.full((n + 1,), 5, dtype=torch.int32, device="cuda")
    offset[:3], offset[3:n] = torch.tensor([0, 0, 2]), 4                     # experts 1, 2 and the last have places
    w = torch.zeros((1, 1, h), device="cuda").expand(n, 1, h)
    _, dw = gpu.topk_expert_product_vjp(x, w, offset, t, want_x=False)
    at = offset.tolist()
    for e in range(n):
        if at[e] == at[e + 1]:
            assert (dw[e] == 0).all(), e
        else:
            part = slice(at[e], at[e + 1])
            terms = t[part].double() * x[part].double()
            # two products and their sum, rounded
            assert ((dw[e, 0].double() - terms.sum(dim=0)).abs() <= 3 * 2.0 ** -24 * terms.abs().sum(dim=0)).all(), e
