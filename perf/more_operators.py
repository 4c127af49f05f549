"""The work that is timed on the experts' feed-forward: the gated block (two projections, the activation and the product) with its
gradients, and products in 8-bit integers with a scale for every token and channel, plain and gated.

Every case is one pass, with `own` false in a plain form of elementary torch operations in 32 bits (in 64 where a value is rounded
to 8 bits), with `own` true through the Python binding.  The sizes are those of the router workloads of this repository (64
experts with k = 2, 128 with k = 8) and generic ones around them; `draw` spreads each kind over its range.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_BYTES = {"f32": 4, "bf16": 2, "f16": 2}
_ACTS = ("silu", "gelu", "gelu_tanh", "relu")
_binding = None


def _lib():
    global _binding
    if _binding is None:
        from paper_2302_01425_amd import binding
        _binding = binding
    return _binding


def _case(op, rows, n, k, h, f, dtype, act="", gather=True, turned=False, kept=False):
    """rows tokens to k of n experts, h -> f.  gather: rows of x are found through the list of places, otherwise they lie in
    expert order.  turned: weights lie with their outputs along the last dimension.  kept: the forward pass left its sums."""
    return dict(op=op, rows=rows, n=n, k=k, h=h, f=f, dtype=dtype, act=act, gather=gather, turned=turned, kept=kept)


def listed():
    return [
        # one token of one request is decoded: a call whose latency counts
        dict(name="gated one token", **_case("gated_fwd", 1, 8, 2, 2048, 1024, "bf16", "silu")),
        # training step of token-choice experts, forward and both kinds of gradients
        dict(name="gated", **_case("gated_fwd", 8192, 32, 2, 2048, 2048, "bf16", "silu")),
        dict(name="gated vjp", **_case("gated_vjp", 8192, 32, 2, 2048, 2048, "bf16", "silu")),
        # the same step where memory allows the sums of the forward pass to be kept; odd sizes, float16
        dict(name="gated vjp kept", **_case("gated_vjp", 4001, 16, 2, 1001, 1515, "f16", "gelu", kept=True)),
        # ragged sizes in single precision, rows already in expert order
        dict(name="gated odd f32", **_case("gated_fwd", 1003, 10, 3, 515, 1001, "f32", "gelu_tanh", gather=False)),
        # a decoding batch through the second projection in 8 bits: the weights are read, little is computed
        dict(name="product i8 decode", **_case("product_i8", 32, 64, 4, 1024, 2048, "bf16", gather=False)),
        # prefill through the first projection of plain experts in 8 bits
        dict(name="product i8", **_case("product_i8", 8192, 32, 2, 2048, 4096, "bf16")),
        # odd widths of rows of bytes
        dict(name="product i8 odd", **_case("product_i8", 3001, 12, 2, 1001, 2003, "f16")),
        # one token and a decoding batch through the gated block in 8 bits
        dict(name="gated i8 one token", **_case("gated_i8", 1, 8, 2, 2048, 1024, "bf16", "silu")),
        dict(name="gated i8 decode", **_case("gated_i8", 64, 128, 8, 2048, 768, "bf16", "silu")),
        # prefill
        dict(name="gated i8", **_case("gated_i8", 8192, 32, 2, 2048, 2048, "bf16", "silu")),
    ]


def _log(rng, lo, hi):
    """A whole number between lo and hi, uniform in its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("gated_fwd", "gated_fwd", "gated_vjp", "product_i8", "product_i8", "gated_i8"))
    eight = op.endswith("i8")
    dtype = rng.choice(("f32", "bf16", "f16"))
    n = _log(rng, 1, 128)
    k = rng.randint(1, min(8, n))
    h, f = _log(rng, 64, 4096), _log(rng, 64, 4096)
    # half of the widths are multiples of 64, as most models have them
    if rng.random() < 0.5:
        h, f = -(-h // 64) * 64, -(-f // 64) * 64
    # no more than the weights and the operations of the largest listed case; float32, whose matrix rate is an eighth of the
    # others', an eighth of the operations
    n = max(k, min(n, (1 << 27) // (h * f)))
    most = (16384 * 2048 * 2048) // (8 if dtype == "f32" and not eight else 1)
    rows = _log(rng, 1, max(1, min(8192, most // (h * f * k))))
    act = "" if op == "product_i8" else rng.choice(_ACTS)
    return _case(op, rows, n, k, h, f, dtype, act, gather=rng.random() < 0.6, turned=not eight and rng.random() < 0.25,
                 kept=op == "gated_vjp" and rng.random() < 0.5)


# ---- inputs ---------------------------------------------------------------------------------------------------------

def _lists(gen, rows, n, k):
    """Places in expert order of tokens whose choices are those of a trained router: some experts are liked by many tokens,
    some by few, none is chosen twice by a token.  source: the pair token * k + choice behind a place; offset: where the places
    of an expert begin."""
    liked = 0.7 * torch.randn((1, n), generator=gen, device="cuda")
    chosen = (torch.randn((rows, n), generator=gen, device="cuda") + liked).topk(k, dim=1).indices.reshape(-1)
    order = torch.sort(chosen, stable=True)
    begin = torch.searchsorted(order.values, torch.arange(n + 1, device="cuda"))
    return order.indices.to(torch.int32).contiguous(), begin.to(torch.int32).contiguous()


def _to_8_bits(x):
    """Rows as 8-bit integers q and scales: x is about q * scale, the largest of a row is 127 away from zero."""
    top = x.double().abs().amax(dim=-1, keepdim=True)
    safe = torch.where(top == 0, torch.ones_like(top), top)
    q = torch.round(127.0 * x.double() / safe).to(torch.int8)
    return q, (top / 127.0).squeeze(-1).float()


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    op, rows, n, k, h, f, dtype = (case[c] for c in ("op", "rows", "n", "k", "h", "f", "dtype"))
    s = {"case": case}

    def randn(shape, scale=1.0):
        return (torch.randn(shape, generator=gen, device="cuda") * scale).to(_TYPES[dtype])

    def weights(scale):
        # drawn expert by expert, so that float32 values of one only are there at a time
        w = torch.empty((n, h, f) if case["turned"] else (n, f, h), dtype=_TYPES[dtype], device="cuda")
        for part in w:
            part.copy_(torch.randn(part.shape, generator=gen, device="cuda") * scale)
        return w.transpose(1, 2) if case["turned"] else w

    def weights_8(scale):
        # quantised once, when a model is loaded
        q = torch.empty((n, f, h), dtype=torch.int8, device="cuda")
        qs = torch.empty((n, f), dtype=torch.float32, device="cuda")
        for e in range(n):
            q[e], qs[e] = _to_8_bits(torch.randn((f, h), generator=gen, device="cuda") * scale)
        return q, qs

    source, s["offset"] = _lists(gen, rows, n, k)
    s["source"] = source if case["gather"] else None
    s["x"] = randn((rows if case["gather"] else rows * k, h))
    size = 1.0 / math.sqrt(h)
    if op.endswith("i8"):
        # a few channels are larger than the others, as behind a norm
        s["x"] *= torch.where(torch.rand(h, generator=gen, device="cuda") < 0.01, 8.0, 1.0).to(_TYPES[dtype])
        s["w"], s["w_scale"] = weights_8(size)
        if op == "gated_i8":
            s["w2"], s["w2_scale"] = weights_8(size)
        return s
    s["w"], s["w2"] = weights(size), weights(size)
    if op == "gated_vjp":
        s["t"] = randn((rows * k, f))
        s["pre"] = None
        if case["kept"]:
            s["pre"] = torch.stack(_sums(s, s["w"], s["w2"]), dim=1).to(_TYPES[dtype])
    return s


# ---- plain forms ----------------------------------------------------------------------------------------------------

def _experts(s):
    """(expert, its places, its rows of x) for every expert that has places."""
    at = s["offset"].tolist()
    for e in range(s["case"]["n"]):
        lo, hi = at[e], at[e + 1]
        if lo < hi:
            row = slice(lo, hi) if s["source"] is None else (s["source"][lo:hi] // s["case"]["k"]).long()
            yield e, slice(lo, hi), row


def _sums(s, *ws):
    """Every place's row through its expert's matrices, in float32."""
    c = s["case"]
    out = [torch.empty((c["rows"] * c["k"], c["f"]), device="cuda") for _ in ws]
    for e, place, row in _experts(s):
        x = s["x"][row].float()
        for o, w in zip(out, ws):
            o[place] = x @ w[e].float().t()
    return out


def _act(act, g):
    """Value and derivative."""
    if act == "silu":
        p = 1.0 / (1.0 + torch.exp(-g))
        return g * p, p * (1.0 + g * (1.0 - p))
    if act == "gelu":
        p = 0.5 * (1.0 + torch.erf(g * math.sqrt(0.5)))
        return g * p, p + g * torch.exp(-0.5 * g * g) * (1.0 / math.sqrt(2.0 * math.pi))
    if act == "gelu_tanh":
        c = math.sqrt(2.0 / math.pi)
        th = torch.tanh(c * (g + 0.044715 * g * g * g))
        return 0.5 * g * (1.0 + th), 0.5 * (1.0 + th) + 0.5 * g * (1.0 - th * th) * c * (1.0 + 3.0 * 0.044715 * g * g)
    pos = g > 0
    return torch.where(pos, g, torch.zeros_like(g)), pos.to(g.dtype)


def _plain_gated(s):
    g, u = _sums(s, s["w"], s["w2"])
    return (_act(s["case"]["act"], g)[0] * u).to(s["x"].dtype)


def _plain_gated_vjp(s):
    c, x = s["case"], s["x"]
    g, u = _sums(s, s["w"], s["w2"]) if s["pre"] is None else (s["pre"][:, 0].float(), s["pre"][:, 1].float())
    value, slope = _act(c["act"], g)
    t = s["t"].float()
    dg, du = t * u * slope, t * value
    dx = torch.empty((c["rows"] * c["k"], c["h"]), dtype=x.dtype, device="cuda")
    dw, dw2 = torch.zeros_like(s["w"]), torch.zeros_like(s["w2"])
    for e, place, row in _experts(s):
        xe = x[row].float()
        dx[place] = (dg[place] @ s["w"][e].float() + du[place] @ s["w2"][e].float()).to(x.dtype)
        dw[e] = (dg[place].t() @ xe).to(x.dtype)
        dw2[e] = (du[place].t() @ xe).to(x.dtype)
    return dx, dw, dw2


def _plain_sums_8(s, q, scale, w, w_scale):
    """Sums of products of 8-bit integers: 1024 of them are exact in float32, and such parts are added as int32."""
    c = s["case"]
    out = torch.empty((c["rows"] * c["k"], c["f"]), device="cuda")
    for e, place, row in _experts(s):
        a = q[row]
        total = torch.zeros((a.shape[0], c["f"]), dtype=torch.int32, device="cuda")
        for i in range(0, c["h"], 1024):
            total += (a[:, i:i + 1024].float() @ w[e, :, i:i + 1024].float().t()).to(torch.int32)
        out[place] = total.float() * scale[row].unsqueeze(1) * w_scale[e]
    return out


def _plain_product_8(s):
    q, scale = _to_8_bits(s["x"])
    return _plain_sums_8(s, q, scale, s["w"], s["w_scale"]).to(s["x"].dtype)


def _plain_gated_8(s):
    q, scale = _to_8_bits(s["x"])
    g = _plain_sums_8(s, q, scale, s["w"], s["w_scale"])
    u = _plain_sums_8(s, q, scale, s["w2"], s["w2_scale"])
    return (_act(s["case"]["act"], g)[0] * u).to(s["x"].dtype)


def run(s):
    c = s["case"]
    op = c["op"]
    if not own:
        return {"gated_fwd": _plain_gated, "gated_vjp": _plain_gated_vjp, "product_i8": _plain_product_8,
                "gated_i8": _plain_gated_8}[op](s)
    b = _lib()
    act = {"": 0, "silu": b.TOPK_ACT_SILU, "gelu": b.TOPK_ACT_GELU, "gelu_tanh": b.TOPK_ACT_GELU_TANH,
           "relu": b.TOPK_ACT_RELU}[c["act"]]
    if op == "gated_fwd":
        return b.topk_expert_gated_fwd(s["x"], s["w"], s["w2"], s["offset"], source=s["source"], k=c["k"], act=act)
    if op == "gated_vjp":
        return b.topk_expert_gated_vjp(s["x"], s["w"], s["w2"], s["offset"], s["t"], source=s["source"], k=c["k"], act=act,
                                       pre=s["pre"])
    # tokens come in 16 or 32 bits and are quantised on the way
    q, scale = b.topk_quantise_rows(s["x"])
    if op == "product_i8":
        return b.topk_expert_product_i8_fwd(q, scale, s["w"], s["w_scale"], s["offset"], source=s["source"], k=c["k"],
                                            dtype=s["x"].dtype)
    return b.topk_expert_gated_i8_fwd(q, scale, s["w"], s["w_scale"], s["w2"], s["w2_scale"], s["offset"], source=s["source"],
                                      k=c["k"], act=act, dtype=s["x"].dtype)


# ---- the definition in 64 bits --------------------------------------------------------------------------------------

def _gate_64(act, g):
    """act(g) and act'(g), each from a form that keeps its digits for large |g|."""
    if act == "silu":
        p, r = torch.special.expit(g), torch.special.expit(-g)
        return g * p, p + g * p * r
    if act == "gelu":
        p = 0.5 * torch.special.erfc(-g / math.sqrt(2.0))
        return g * p, p + g * torch.exp(-g.square() / 2) / math.sqrt(2 * math.pi)
    if act == "gelu_tanh":
        # (1 + tanh z) / 2 = expit(2 z)
        z2 = math.sqrt(8.0 / math.pi) * (g + 0.044715 * g.pow(3))
        p, r = torch.special.expit(z2), torch.special.expit(-z2)
        return g * p, p + g * p * r * math.sqrt(8.0 / math.pi) * (1 + 0.134145 * g.square())
    return g.clamp(min=0.0), torch.where(g > 0, 1.0, 0.0).double()


def exact(case, seed):
    s = prepare(case, seed)
    op, k, f = case["op"], case["k"], case["f"]
    at = s["offset"].cpu().numpy()
    pairs = case["rows"] * k
    token = torch.arange(pairs, device="cuda") if s["source"] is None else torch.div(s["source"].long(), k, rounding_mode="floor")
    x = s["x"].double()
    if op.endswith("i8"):
        top = x.abs().max(dim=1).values
        x = torch.where(top[:, None] > 0, torch.round(x * 127.0 / top[:, None]), torch.zeros_like(x))
        unit = top / 127.0
    names = ("w",) if op == "product_i8" else ("w", "w2")
    out = torch.zeros((pairs, f), dtype=torch.float64, device="cuda")
    dx = dw = None
    if op == "gated_vjp":
        out = None
        dx = torch.zeros((pairs, case["h"]), dtype=torch.float64, device="cuda")
        dw = [torch.zeros(s["w"].shape, dtype=torch.float64, device="cuda") for _ in names]
    for e in np.flatnonzero(np.diff(at)):
        e = int(e)
        part = slice(int(at[e]), int(at[e + 1]))
        xe = x[token[part]]
        ws = [s[name][e].double().contiguous() for name in names]
        if op == "gated_vjp" and case["kept"]:
            sums = [s["pre"][part, i].double() for i in range(2)]
        else:
            sums = [torch.mm(xe, w.t().contiguous()) for w in ws]
        if op.endswith("i8"):
            sums = [v * unit[token[part], None] * s[name + "_scale"][e].double() for v, name in zip(sums, names)]
        if op == "product_i8":
            out[part] = sums[0]
            continue
        value, slope = _gate_64(case["act"], sums[0])
        if op != "gated_vjp":
            out[part] = value * sums[1]
            continue
        t = s["t"][part].double()
        ds = (t * sums[1] * slope, t * value)
        dx[part] = torch.mm(ds[0], ws[0]) + torch.mm(ds[1], ws[1])
        for i in range(2):
            dw[i][e] = torch.mm(ds[i].t().contiguous(), xe)
    return out if dx is None else (dx, dw[0], dw[1])


def work(case):
    """Bytes: every input read once, every output written once (of the experts' weights those that have rows, as many as
    independent choices would hit).  Operations: those of the products."""
    op, rows, n, k, h, f = (case[c] for c in ("op", "rows", "n", "k", "h", "f"))
    b = _BYTES[case["dtype"]]
    pairs = rows * k
    hit = n * (1.0 - (1.0 - 1.0 / n) ** pairs)
    lists = 4 * (n + 1) + (4 * pairs if case["gather"] else 0)
    x = (rows if case["gather"] else pairs) * h * b
    if op.endswith("i8"):
        times = 1 if op == "product_i8" else 2
        return {"bytes": x + times * hit * (h * f + 4 * f) + pairs * f * b + lists, "flops": 2.0 * times * pairs * h * f}
    if op == "gated_fwd":
        return {"bytes": x + 2 * hit * h * f * b + pairs * f * b + lists, "flops": 4.0 * pairs * h * f}
    kept = 2 * pairs * f * b if case["kept"] else 0
    return {"bytes": x + 2 * hit * h * f * b + pairs * f * b + kept + pairs * h * b + 2 * n * h * f * b + lists,
            "flops": (8.0 if case["kept"] else 12.0) * pairs * h * f}
