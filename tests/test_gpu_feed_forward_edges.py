"""The experts' feed-forward on the GPU where test_gpu_feed_forward.py does not reach: rows in 8 bits up to the largest numbers, scales
of any size, long float32 sums, and the kernels that only calls of certain sizes take.  Comparisons and tolerances as there."""
import numpy as np
import pytest

from tests import test_gpu_feed_forward as base
from tests.test_gpu_experts import HALF, TINY, U, host, put, rounded

pytestmark = pytest.mark.gpu
DTYPES = ("float32", "bfloat16", "float16")
LARGEST = {"float32": (2.0 - 2.0 ** -23) * 2.0 ** 127, "bfloat16": (2.0 - 2.0 ** -7) * 2.0 ** 127, "float16": 65504.0}


@pytest.fixture(scope="module")
def gpu():
    import torch
    from paper_2302_01425_amd import binding
    assert torch.cuda.is_available()
    binding.load()
    return binding


# ---- rows in 8 bits ---------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("h", [7, 64, 513, 2048, 20003])
@pytest.mark.parametrize("dtype", DTYPES)
def test_quantise_beside_halves_of_large_rows(gpu, h, dtype):
    """Quotients at a half and a few steps of the type beside it, in rows whose largest magnitude is up to the type's largest number:
    127 x and (H + 1/2) a are exact in float64, and compared."""
    r = np.random.default_rng(h)
    m = 300
    low, high = (95, 128) if dtype != "float16" else (10, 16)
    a = rounded(np.minimum(np.ldexp(1.0 + r.random(m), r.integers(low, high, m)), LARGEST[dtype]), dtype)
    a[0] = LARGEST[dtype]
    half = r.integers(0, 127, (m, h)) + 0.5
    steps = r.integers(-3, 4, (m, h))
    x = rounded(half * a[:, None] / 127.0, dtype)
    x = np.clip(rounded(x * (1.0 + steps * 2 * HALF[dtype]), dtype), 0.0, a[:, None])
    x[:, ::5] = a[:, None] / 2                              # quotient 63.5
    x *= r.choice([-1.0, 1.0], (m, h))
    x[:, h // 2] = a
    assert np.isfinite(x).all() and np.array_equal(x, rounded(x, dtype))
    n = np.floor(127.0 * np.abs(x) / a[:, None] + 0.25)                     # the half beside which it lies, or none near
    whole = np.rint(127.0 * np.abs(x) / a[:, None])
    gap = 127.0 * np.abs(x) - (n + 0.5) * a[:, None]
    near = np.abs(127.0 * np.abs(x) / a[:, None] - (n + 0.5)) < 0.1
    want = np.where(near, np.where(gap > 0, n + 1, np.where(gap < 0, n, 2 * np.ceil(n / 2))), whole) * np.sign(x)
    q, scale = gpu.topk_quantise_rows(put(x, dtype))
    assert np.array_equal(host(q), want)
    assert np.array_equal(host(scale).astype(np.float32), a.astype(np.float32) / np.float32(127.0))


# rows, k, n, h, f: by vector sums, 32 rows of half the columns and of all, 64 rows, 128 x 128, 256 x 256
SCALED = [(1, 2, 4, 64, 40), (2, 2, 4, 4100, 24), (256, 2, 8, 512, 448), (300, 2, 2, 129, 1141), (2600, 2, 4, 264, 520),
          (3000, 2, 8, 1040, 2176), (20, 2, 3, 9, 15)]


@pytest.mark.parametrize("rows,k,n,h,f", SCALED)
@pytest.mark.parametrize("dtype", DTYPES)
def test_scales_of_any_size_in_8_bits(gpu, rows, k, n, h, f, dtype):
    """Scales of rows and channels whose product is moderate, while either is near one end of float32: nothing between may leave its
    range.  Two products and the sum's conversion are rounded: (HALF + 4 u) of the exact value; for the gated block three of either
    sum and their product: (HALF + 8 u)."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(rows + h)
    dt = getattr(torch, dtype)
    source, offset, at = base.large_lists(gpu, rows, k, n, g)
    q, wg, wu = (torch.randint(-128, 128, s, generator=g, device="cuda", dtype=torch.int8) for s in ((rows, h), (n, f, h), (n, f, h)))

    def scale(shape, power):
        return (torch.rand(shape, generator=g, device="cuda") + 1.0) * 2.0 ** power

    for rows_power, channels_power in ((110, -126), (122, -138), (-126, 110), (-134, 118), (28, -44), (-44, 28)):
        xs, gs, us = scale((rows,), rows_power), scale((n, f), channels_power), scale((n, f), channels_power)
        xs[::5] *= 2.0 ** -3
        xs[1::5] = 0.0                                      # (a row of zeros)
        xs[2::5] *= -1.0
        gs[:, ::3] *= -1.0
        print("case", rows, k, n, h, f, dtype, rows_power, flush=True)
        out = gpu.topk_expert_product_i8_fwd(q, xs, wg, gs, offset, source, k, dt)
        both = gpu.topk_expert_gated_i8_fwd(q, xs, wg, gs, wu, us, offset, source, k, gpu.TOPK_ACT_RELU, dt)
        for e in range(n):
            part = slice(at[e], at[e + 1])
            row = (source[part] // k).long()
            xe = q[row].double()
            a, b = ((xe @ w[e].double().t().contiguous()) * xs[row].double()[:, None] * s[e].double() for w, s in ((wg, gs), (wu, us)))
            c = a.clamp(min=0) * b
            assert (out[part].double() - a).abs().le((HALF[dtype] + 4 * U) * a.abs() + TINY[dtype]).all(), e
            assert (both[part].double() - c).abs().le((HALF[dtype] + 8 * U) * c.abs() + TINY[dtype]).all(), e


# ---- float32 sums -----------------------------------------------------------------------------------------------------

# rows and columns: four rows at a time; 32 rows of half the columns, of all; 64 rows
LONG = [(4, 64), (64, 64), (256, 768), (256, 1088), (1024, 1024)]


def long_rows(m, h, big, seed):
    """Ones, and 2^27 at `big`: additions of the others to it lose them, at most 8 each.  A part of 128 terms and the additions of at
    most h / 128 parts and of a few wavefronts' sums are hence off by 128 + 8 (h / 128 + 8)."""
    import torch
    x = torch.ones((m, h), device="cuda")
    x[:, big] = 2.0 ** 27
    return x, 2.0 ** 27 + h - 1, 128 + 8 * (h // 128 + 8)


@pytest.mark.parametrize("rows,f", LONG)
@pytest.mark.parametrize("big", [0, 4100, 16383])
def test_long_sums_of_float32(gpu, rows, f, big):
    """max(g, 0) u with u = 1: g a sum of 16384 terms, W contiguous in k and with one row per k."""
    import torch
    h = 16384
    x, want, most = long_rows(rows, h, big, 0)
    off = torch.tensor([0, rows], dtype=torch.int32, device="cuda")
    wg, wu = torch.ones((1, f, h), device="cuda"), torch.zeros((1, f, h), device="cuda")
    wu[:, :, 7] = 1.0
    for turned in (False, True):
        if turned:
            wg, wu = (w.transpose(1, 2).contiguous().transpose(1, 2) for w in (wg, wu))
        print("case", rows, f, big, turned, flush=True)
        out = gpu.topk_expert_gated_fwd(x, wg, wu, off, act=gpu.TOPK_ACT_RELU)
        off_by = float((out.double() - want).abs().max())
        assert off_by <= most, (off_by, most)


@pytest.mark.parametrize("rows,h", [(1, 64), (32, 64), (256, 2176), (1024, 2048)])
@pytest.mark.parametrize("big", [0, 4100, 16383])
def test_long_sums_of_float32_in_dx(gpu, rows, h, big):
    """Kept sums of 1: dg = t, times ones."""
    import torch
    f = 16384
    t, want, most = long_rows(rows, f, big, 0)
    off = torch.tensor([0, rows], dtype=torch.int32, device="cuda")
    x, pre = torch.ones((rows, h), device="cuda"), torch.ones((rows, 2, f), device="cuda")
    wg, wu = torch.ones((1, f, h), device="cuda"), torch.zeros((1, f, h), device="cuda")
    for turned in (False, True):
        if turned:
            wg, wu = (w.transpose(1, 2).contiguous().transpose(1, 2) for w in (wg, wu))
        print("case", rows, h, big, turned, flush=True)
        dx = gpu.topk_expert_gated_vjp(x, wg, wu, off, t, act=gpu.TOPK_ACT_RELU, pre=pre, want_w=False)[0]
        off_by = float((dx.double() - want).abs().max())
        assert off_by <= most, (off_by, most)


# ---- kernels that only some sizes take ----------------------------------------------------------------------------------

@pytest.mark.parametrize("rows,k,n,h,f", [(8192, 2, 8, 1032, 1544), (8192, 2, 8, 1536, 1536)])
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
def test_dx_of_large_tiles(gpu, rows, k, n, h, f, dtype):
    """dx by tiles of 256 x 256 (192 of them at least): several tiles of columns, whose sums begin at different steps, a last step and a
    last tile that are not whole, and whole ones; weights contiguous in either direction."""
    base.test_large_whole_numbers(gpu, rows, k, n, h, f, dtype)


@pytest.mark.parametrize("rows,k,n,h,f", [(3000, 2, 8, 1040, 2176), (2100, 2, 6, 2064, 2048), (256, 2, 8, 512, 896), (256, 2, 8, 512, 448)])
def test_8_bits_by_size(gpu, rows, k, n, h, f):
    """256 x 256 with a last step that is not whole; 32 rows of all columns, plain (f 896) and gated (448)."""
    base.test_large_products_of_8_bits(gpu, rows, k, n, h, f)


@pytest.mark.parametrize("rows,k,n,h,f", [(8, 2, 4, 4096, 1024), (8, 2, 4, 4096, 512)])
@pytest.mark.parametrize("dtype", DTYPES)
def test_few_rows_of_8_bits_in_turns(gpu, rows, k, n, h, f, dtype):
    """k shared by wavefronts that take two turns of columns, plain (f 1024) and gated (512)."""
    base.test_products_of_8_bits(gpu, rows, k, n, h, f, dtype)


@pytest.mark.parametrize("rows,k,n,h,f,dtype", [(1, 2, 8, 2048, 1024, "bfloat16"), (1, 2, 8, 2048, 1024, "float16"),
                                                (1, 2, 2, 2049, 2201, "bfloat16"), (1, 2, 2, 2049, 2201, "float16"),
                                                (4, 2, 4, 1100, 1501, "float32"), (4, 2, 4, 1027, 702, "float32"),
                                                (256, 2, 8, 2049, 150, "bfloat16"), (256, 2, 8, 2049, 150, "float16")])
def test_few_rows_by_size(gpu, rows, k, n, h, f, dtype):
    """k shared by the wavefronts in 16 bits, in one and two turns of columns; in float32 in four and two; 32 rows of half the columns
    where W's rows begin anywhere."""
    base.test_whole_numbers(gpu, rows, k, n, h, f, dtype)


@pytest.mark.parametrize("rows,k,n,h,f", [(130, 2, 16, 1001, 1001), (400, 2, 40, 520, 2048), (300, 2, 12, 776, 1032)])
@pytest.mark.parametrize("dtype", DTYPES)
def test_many_experts_of_few_rows(gpu, rows, k, n, h, f, dtype):
    """32 rows of all columns: float32 at any alignment (512 tiles), more than 1024 tiles of experts with at most 32 places, also where W
    has one row per k; 50 places per expert (792 tiles: 64 rows)."""
    base.test_large_whole_numbers(gpu, rows, k, n, h, f, dtype)
