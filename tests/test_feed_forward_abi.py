"""What the entry points of the experts' feed-forward refuse before anything is enqueued (no GPU is needed)."""
import ctypes
import os

import pytest


@pytest.fixture(scope="module")
def lib():
    from paper_2302_01425_amd import binding
    if not os.path.exists(binding.LIB_PATH):
        from paper_2302_01425_amd import build
        build.build_library(verbose=False)
    return binding.load()


ONE = ctypes.c_void_p(256)          # never dereferenced: validation happens first
GATED = dict(x=ONE, x_stride=8, m=4, w_gate=ONE, w_up=ONE, w_expert=32, w_out=8, w_in=1, offset=ONE, source=ONE, k=2, slots=8,
             n=3, h=8, f=4, type=0, act=0)
EIGHT = dict(x=ONE, x_stride=8, m=4, x_scale=ONE, w=ONE, w_scale=ONE, w_expert=32, w_out=8, offset=ONE, source=ONE, k=2, slots=8,
             n=3, h=8, f=4, out_type=0, out=ONE)
MOST = 1 << 31
BAD_LISTS = [dict(n=0), dict(n=1025), dict(h=0), dict(f=0), dict(h=MOST), dict(f=MOST), dict(slots=-1), dict(slots=MOST), dict(m=-1),
             dict(m=MOST), dict(k=0), dict(k=MOST), dict(x_stride=-1), dict(w_expert=-1), dict(w_out=-1), dict(source=None)]


def gated_fwd(lib, out=ONE, pre=None, **change):
    return lib.topk_expert_gated_fwd(*(dict(GATED, **change)).values(), out, pre, None)


def gated_vjp(lib, pre=None, t=ONE, t_stride=4, dx=ONE, dwg=ONE, dwu=ONE, scratch=ONE, size=1 << 20, **change):
    return lib.topk_expert_gated_vjp(*(dict(GATED, **change)).values(), pre, t, t_stride, dx, dwg, dwu, scratch, size, None)


def product(lib, **change):
    a = dict(EIGHT, **change)
    return lib.topk_expert_product_i8_fwd(*(a[c] for c in ("x", "x_stride", "m", "x_scale", "w", "w_expert", "w_out", "w_scale", "offset",
                                                           "source", "k", "slots", "n", "h", "f", "out_type", "out")), None)


def gated_i8(lib, w_up=ONE, up_scale=ONE, act=0, **change):
    a = dict(EIGHT, **change)
    return lib.topk_expert_gated_i8_fwd(a["x"], a["x_stride"], a["m"], a["x_scale"], a["w"], a["w_scale"], w_up, up_scale,
                                        *(a[c] for c in ("w_expert", "w_out", "offset", "source", "k", "slots", "n", "h", "f",
                                                         "out_type")), act, a["out"], None)


@pytest.mark.parametrize("change", BAD_LISTS)
def test_lists_and_shapes(lib, change):
    assert gated_fwd(lib, **change) == -1
    assert gated_vjp(lib, **change) == -1
    assert product(lib, **change) == -1
    assert gated_i8(lib, **change) == -1


def test_gated(lib):
    for change in (dict(type=3), dict(type=-1), dict(act=4), dict(act=-1), dict(w_in=2), dict(w_in=-1)):
        assert gated_fwd(lib, **change) == -1 and gated_vjp(lib, **change) == -1
    for change in (dict(x=None), dict(w_gate=None), dict(w_up=None), dict(offset=None)):
        assert gated_fwd(lib, **change) == -2 and gated_vjp(lib, **change) == -2
    assert gated_fwd(lib, out=None) == -2
    assert gated_vjp(lib, t=None) == -2
    assert gated_vjp(lib, t_stride=-1) == -1
    assert gated_vjp(lib, dwg=None) == -2 and gated_vjp(lib, dwu=None) == -2
    assert gated_vjp(lib, dx=None, dwg=None, dwu=None) == -2
    assert gated_vjp(lib, scratch=None) == -4 and gated_vjp(lib, scratch=ctypes.c_void_p(264)) == -1
    assert gated_fwd(lib, slots=0) == 0
    assert gated_vjp(lib, slots=0, dwg=None, dwu=None) == 0


def test_scratch(lib):
    size = lib.topk_expert_gated_vjp_bytes
    # two halves of whole 16-byte parts per place
    assert size(8, 4, 0) == 8 * 2 * 4 * 4 and size(8, 5, 0) == 8 * 2 * 8 * 4
    assert size(8, 5, 1) == 8 * 2 * 8 * 2 and size(3, 9, 2) == 3 * 2 * 16 * 2
    assert size(0, 4, 0) == 0 and size(-1, 4, 0) == 0 and size(8, 0, 0) == 0 and size(8, 4, 3) == 0
    assert size(MOST - 1, MOST - 1, 0) == 2 ** 64 - 1                                 # (2^65 bytes: more than there can be)
    assert gated_vjp(lib, size=size(8, 4, 0) - 1) == -4


def test_eight(lib):
    for call in (product, gated_i8):
        assert call(lib, h=131072) == -1 and call(lib, out_type=3) == -1 and call(lib, out_type=-1) == -1
        for change in (dict(x=None), dict(x_scale=None), dict(w=None), dict(w_scale=None), dict(offset=None), dict(out=None)):
            assert call(lib, **change) == -2, change
        assert call(lib, slots=0) == 0
    assert gated_i8(lib, w_up=None) == -2 and gated_i8(lib, up_scale=None) == -2
    assert gated_i8(lib, act=4) == -1 and gated_i8(lib, act=-1) == -1


def test_quantise(lib):
    q = lib.topk_quantise_rows
    assert q(ONE, 8, -1, 8, 0, ONE, ONE, None) == -1 and q(ONE, 8, MOST, 8, 0, ONE, ONE, None) == -1
    assert q(ONE, 8, 4, 0, 0, ONE, ONE, None) == -1 and q(ONE, 8, 4, MOST, 0, ONE, ONE, None) == -1
    assert q(ONE, -1, 4, 8, 0, ONE, ONE, None) == -1 and q(ONE, 8, 4, 8, 3, ONE, ONE, None) == -1
    assert q(None, 8, 4, 8, 0, ONE, ONE, None) == -2 and q(ONE, 8, 4, 8, 0, None, ONE, None) == -2
    assert q(ONE, 8, 4, 8, 0, ONE, None, None) == -2 and q(None, 8, 0, 8, 0, None, None, None) == 0


def test_binding_refuses_cpu_tensors(lib):
    import torch
    from paper_2302_01425_amd import binding as b
    x, w, o = torch.zeros(2, 8), torch.zeros(1, 4, 8), torch.zeros(2, dtype=torch.int32)
    for call in (lambda: b.topk_expert_gated_fwd(x, w, w, o), lambda: b.topk_expert_gated_vjp(x, w, w, o, x),
                 lambda: b.topk_quantise_rows(x),
                 lambda: b.topk_expert_product_i8_fwd(x.char(), x[:, 0], w.char(), w[..., 0], o),
                 lambda: b.topk_expert_gated_i8_fwd(x.char(), x[:, 0], w.char(), w[..., 0], w.char(), w[..., 0], o)):
        with pytest.raises(b.TopkError):
            call()
