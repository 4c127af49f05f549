"""The experts' feed-forward on the GPU at its edges: rows in 8 bits up to the largest numbers."""
import numpy as np
import pytest

from tests.test_gpu_experts import HALF, host, put, rounded

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
