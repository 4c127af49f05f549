"""The work that is timed on the operators behind a router: choosing experts, the places of the chosen pairs in expert
order, the experts' products over these ragged groups, and the weighted sum back per token.

Every case is one call, with `own` false in a plain form of elementary torch operations in 32 bits (in 64 where scores
are compared), with `own` true through the Python binding.  The sizes are those of the router workloads of this
repository (16384 x 64 with k = 2, 32768 x 128 with k = 8) and generic ones around them; `draw` spreads each kind over
its range.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_BYTES = {"f32": 4, "bf16": 2, "f16": 2}
_binding = None


def _lib():
    global _binding
    if _binding is None:
        from paper_2302_01425_amd import binding
        _binding = binding
    return _binding


def _route(op, rows, n, k, dtype, score, renorm, bias=False, groups=1, keep=1, top=1, padded=0.0):
    return dict(op=op, rows=rows, n=n, k=k, dtype=dtype, score=score, renorm=renorm, bias=bias, groups=groups,
                keep=keep, top=top, padded=padded)


def _map(rows, n, k, capacity=0, padded=0.0):
    return dict(op="map", rows=rows, n=n, k=k, capacity=capacity, padded=padded)


def _product(op, rows, n, k, h, ho, dtype, gather=True):
    return dict(op=op, rows=rows, n=n, k=k, h=h, ho=ho, dtype=dtype, gather=gather)


def _combine(op, rows, n, k, h, dtype, padded=0.0):
    return dict(op=op, rows=rows, n=n, k=k, h=h, dtype=dtype, padded=padded)


def listed():
    return [
        # one token of one request is decoded: a call whose latency counts
        dict(name="route one token", **_route("route_fwd", 1, 64, 2, "f32", "softmax", True)),
        # training step of the token-choice router of this repository's headline workload, a few padded tokens
        dict(name="route", **_route("route_fwd", 16384, 64, 2, "f32", "softmax", True, padded=0.02)),
        # prefill with many small experts: sigmoid scores, balance bias, groups
        dict(name="route groups", **_route("route_fwd", 8192, 256, 8, "bf16", "sigmoid", True, bias=True, groups=8, keep=4,
                                           top=2)),
        # backward pass of a router that keeps the plain probabilities: every logit has a gradient
        dict(name="route vjp", **_route("route_vjp", 32768, 128, 8, "f32", "softmax", False)),
        # places of a decoding batch of 64 requests
        dict(name="map decode", **_map(64, 64, 2)),
        # places of a training batch, with padded tokens and a capacity per expert
        dict(name="map", **_map(32768, 128, 8, capacity=2560, padded=0.02)),
        # a decoding batch through the experts' first product: the weights are read, little is computed
        dict(name="product decode", **_product("product_fwd", 32, 64, 4, 2048, 1024, "bf16")),
        # training step: forward, and both gradients of the same product
        dict(name="product", **_product("product_fwd", 8192, 32, 2, 2048, 4096, "bf16")),
        dict(name="product vjp", **_product("product_vjp", 8192, 32, 2, 2048, 4096, "bf16")),
        # ragged sizes in single precision, second product (rows already in expert order)
        dict(name="product odd f32", **_product("product_vjp", 1003, 10, 3, 515, 1001, "f32", gather=False)),
        # the sum back of a training batch, padded tokens left out
        dict(name="combine", **_combine("combine_fwd", 16384, 64, 2, 2048, "bf16", padded=0.02)),
        # its backward pass, an odd width, more choices
        dict(name="combine vjp", **_combine("combine_vjp", 8191, 128, 8, 1001, "f16")),
    ]


def _log(rng, lo, hi):
    """A whole number between lo and hi, uniform in its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("route_fwd", "route_fwd", "route_vjp", "map", "product_fwd", "product_fwd", "product_vjp",
                     "combine_fwd", "combine_vjp"))
    dtype = rng.choice(("f32", "bf16", "f16"))
    padded = rng.choice((0.0, 0.02, 0.3))
    if op in ("route_fwd", "route_vjp"):
        groups = rng.choice((1, 1, 2, 4, 8)) if op == "route_fwd" else 1
        n = groups * _log(rng, 4, 512 // groups)
        keep = rng.randint(1, groups)
        top = rng.choice((1, 2)) if groups > 1 else 1
        k = rng.randint(1, max(1, min(16, n // groups * keep)))
        rows = _log(rng, 1, min(32768, (1 << 22) // n))
        return _route(op, rows, n, k, dtype, rng.choice(("softmax", "sigmoid")), rng.random() < 0.6,
                      bias=op == "route_fwd" and rng.random() < 0.5, groups=groups, keep=keep, top=top,
                      padded=padded if op == "route_fwd" else 0.0)
    n = _log(rng, 4, 256)
    k = rng.randint(1, min(8, n))
    if op == "map":
        rows = _log(rng, 1, 32768)
        return _map(rows, n, k, capacity=rng.choice((0, 0, 1 + rows * k // n)), padded=padded)
    if op.startswith("combine"):
        h = _log(rng, 64, 8192)
        return _combine(op, _log(rng, 1, max(1, min(32768, (1 << 26) // (h * k)))), n, k, h, dtype, padded=padded)
    n = _log(rng, 4, 128)
    k = min(k, n)
    h, ho = _log(rng, 64, 4096), _log(rng, 64, 4096)
    # no more than the weights (in float32) and the operations of the largest listed case; float32, whose matrix rate
    # is an eighth of the others', an eighth of the operations
    n = max(k, min(n, (1 << 28) // (h * ho)))
    most = (16384 * 2048 * 4096) // (8 if dtype == "f32" else 1)
    rows = _log(rng, 1, max(1, min(8192, most // (h * ho * k))))
    return _product(op, rows, n, k, h, ho, dtype, gather=rng.random() < 0.6)


# ---- inputs ---------------------------------------------------------------------------------------------------------

def _choices(gen, rows, n, k, padded):
    """Chosen experts as a trained router gives them: some are liked by many tokens, some by few; no expert twice in a
    row.  A share of the rows is padding (-1)."""
    liked = 0.7 * torch.randn((1, n), generator=gen, device="cuda")
    idx = (torch.randn((rows, n), generator=gen, device="cuda") + liked).topk(k, dim=1).indices.to(torch.int32)
    if padded > 0.0:
        idx[torch.rand(rows, generator=gen, device="cuda") < padded] = -1
    return idx.contiguous()


def _places(idx, n, capacity):
    """slot, source, offset, load in plain form: a stable sort of the pairs by expert."""
    rows, k = idx.shape
    pairs = rows * k
    e = idx.reshape(-1).long()
    e = torch.where((e >= 0) & (e < n), e, torch.full_like(e, n))
    order = torch.sort(e, stable=True)
    ends = torch.searchsorted(order.values, torch.arange(n, device=e.device), right=True)
    load = torch.diff(ends, prepend=ends.new_zeros(1))
    kept = load if capacity <= 0 else load.clamp(max=capacity)
    offset = torch.cat((kept.new_zeros(1), kept.cumsum(0)))
    rank = torch.arange(pairs, device=e.device) - torch.cat((ends - load, ends[-1:]))[order.values]
    there = (order.values < n) & (rank < torch.cat((kept, kept.new_zeros(1)))[order.values])
    place = offset[order.values] + rank
    slot = torch.empty(pairs, dtype=torch.int32, device=e.device)
    slot[order.indices] = torch.where(there, place, torch.full_like(place, -1)).to(torch.int32)
    # places of pairs that are out go to a spare last element
    source = torch.full((pairs + 1,), -1, dtype=torch.int32, device=e.device)
    source[torch.where(there, place, torch.full_like(place, pairs))] = order.indices.to(torch.int32)
    source = torch.where(torch.arange(pairs, device=e.device) < offset[-1], source[:pairs], -1).to(torch.int32)
    return slot.reshape(rows, k), source, offset.to(torch.int32), load.to(torch.int32)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    op, rows, n, k = case["op"], case["rows"], case["n"], case["k"]
    s = {"case": case}

    def randn(shape, dtype="f32", scale=1.0):
        # drawn in halves of a large array's memory at most: float32 only for one leading index at a time
        out = torch.empty(shape, dtype=_TYPES[dtype], device="cuda")
        parts = out if out.dim() == 3 else out.unsqueeze(0)
        for part in parts:
            part.copy_(torch.randn(part.shape, generator=gen, device="cuda") * scale)
        return out

    if op.startswith("route"):
        liked = torch.randn((1, n), generator=gen, device="cuda")
        logits = torch.randn((rows, n), generator=gen, device="cuda") * 1.5 + liked
        if case["padded"] > 0.0:
            logits[torch.rand(rows, generator=gen, device="cuda") < case["padded"]] = -math.inf
        s["logits"] = logits.to(_TYPES[case["dtype"]]).contiguous()
        s["bias"] = 0.1 * torch.randn(n, generator=gen, device="cuda") if case["bias"] else None
        if op == "route_vjp":
            s["idx"] = _plain_route(case, s["logits"], s["bias"])[0]
            s["t"] = randn((rows, k))
        return s
    idx = _choices(gen, rows, n, k, case.get("padded", 0.0))
    if op == "map":
        s["idx"] = idx
        return s
    s["slot"], s["source"], s["offset"], _ = _places(idx, n, 0)
    if op.startswith("combine"):
        h, dtype = case["h"], case["dtype"]
        s["y"] = randn((rows * k, h), dtype)
        s["val"] = torch.softmax(randn((rows, k)), dim=1)
        if op == "combine_vjp":
            s["t"] = randn((rows, h), dtype)
            # rows behind the last place are left as they were: the program keeps the buffer
            s["dy"] = torch.zeros_like(s["y"])
        return s
    h, ho, dtype = case["h"], case["ho"], case["dtype"]
    s["x"] = randn((rows if case["gather"] else rows * k, h), dtype)
    s["w"] = randn((n, ho, h), dtype, 1.0 / math.sqrt(h))
    if op == "product_vjp":
        s["t"] = randn((rows * k, ho), dtype)
    return s


# ---- plain forms ----------------------------------------------------------------------------------------------------

def _scores(case, logits, dtype):
    l = logits.to(dtype)
    l = torch.where(torch.isnan(l), torch.full_like(l, -math.inf), l)
    if case["score"] == "sigmoid":
        return 1.0 / (1.0 + torch.exp(-l))
    top = l.max(dim=1, keepdim=True).values
    e = torch.exp(l - torch.where(torch.isinf(top), torch.zeros_like(top), top))
    total = e.sum(dim=1, keepdim=True)
    return e / torch.where(total == 0, torch.ones_like(total), total)


def _plain_route(case, logits, bias):
    rows, n, k = case["rows"], case["n"], case["k"]
    groups, keep = case["groups"], case["keep"]
    # scores next to each other decide who is chosen: in 64 bits
    c = _scores(case, logits, torch.float64)
    # without a bias the order of the scores is the logits' own
    order = logits.double() if bias is None else c + bias.double()
    out = torch.isneginf(logits.double()) | torch.isnan(logits.double())
    if bias is not None:
        out = out | torch.isneginf(bias) | torch.isnan(bias)
    order = torch.where(out, torch.full_like(order, -math.inf), order)
    if groups > 1:
        by = order if case["top"] == 1 or bias is not None else torch.where(out, torch.full_like(c, -math.inf), c)
        best = torch.sort(by.reshape(rows, groups, n // groups), dim=2, descending=True).values[..., :case["top"]]
        # a group with one expert left has that one's score
        best[..., 1:] = torch.where(torch.isneginf(best[..., 1:]), torch.zeros_like(best[..., 1:]), best[..., 1:])
        ranked = torch.sort(best.sum(dim=2), dim=1, descending=True, stable=True).indices[:, :keep]
        stays = torch.zeros((rows, groups), dtype=torch.bool, device=logits.device).scatter_(1, ranked, True)
        order = torch.where(stays.repeat_interleave(n // groups, dim=1), order, torch.full_like(order, -math.inf))
    chosen = torch.sort(order, dim=1, descending=True, stable=True)
    empty = torch.isneginf(chosen.values[:, :k])
    idx = chosen.indices[:, :k]
    val = torch.where(empty, torch.zeros_like(idx, dtype=torch.float32), c.float().gather(1, idx))
    if case["renorm"]:
        total = val.sum(dim=1, keepdim=True)
        val = val / torch.where(total == 0, torch.ones_like(total), total)
    return torch.where(empty, torch.full_like(idx, -1), idx).to(torch.int32), val


def _plain_route_vjp(case, logits, idx, t):
    s = _scores(case, logits, torch.float32)
    there = idx >= 0
    at = torch.where(there, idx, torch.zeros_like(idx)).long()
    chosen = torch.where(there, s.gather(1, at), torch.zeros_like(t))
    ds = torch.where(there, t, torch.zeros_like(t))
    if case["renorm"]:
        total = chosen.sum(dim=1, keepdim=True)
        total = torch.where(total == 0, torch.ones_like(total), total)
        ds = torch.where(there, (ds - (ds * chosen).sum(dim=1, keepdim=True) / total) / total, torch.zeros_like(ds))
    full = torch.zeros_like(s).scatter_add_(1, at, ds)
    if case["score"] == "sigmoid":
        grad = full * s * (1.0 - s)
    else:
        grad = s * (full - (full * s).sum(dim=1, keepdim=True))
    return grad.to(logits.dtype)


def _plain_product(case, x, w, offset, source):
    at = offset.tolist()
    out = torch.empty((case["rows"] * case["k"], case["ho"]), dtype=x.dtype, device=x.device)
    for e in range(case["n"]):
        lo, hi = at[e], at[e + 1]
        if lo == hi:
            continue
        xe = x[(source[lo:hi] // case["k"]).long()] if case["gather"] else x[lo:hi]
        out[lo:hi] = (xe.float() @ w[e].float().t()).to(x.dtype)
    return out


def _plain_product_vjp(case, x, w, offset, source, t):
    at = offset.tolist()
    dx = torch.empty((case["rows"] * case["k"], case["h"]), dtype=x.dtype, device=x.device)
    dw = torch.zeros_like(w)
    for e in range(case["n"]):
        lo, hi = at[e], at[e + 1]
        if lo == hi:
            continue
        xe = x[(source[lo:hi] // case["k"]).long()] if case["gather"] else x[lo:hi]
        te = t[lo:hi].float()
        dx[lo:hi] = (te @ w[e].float()).to(x.dtype)
        dw[e] = (te.t() @ xe.float()).to(w.dtype)
    return dx, dw


def _plain_combine(y, slot, val):
    out = torch.zeros((slot.shape[0], y.shape[1]), dtype=torch.float32, device=y.device)
    for j in range(slot.shape[1]):
        there = slot[:, j:j + 1] >= 0
        part = y[slot[:, j].clamp(min=0).long()].float() * val[:, j:j + 1]
        out += torch.where(there, part, torch.zeros_like(part))
    return out.to(y.dtype)


def _plain_combine_vjp(y, slot, val, t, dy):
    tf = t.float()
    dval = torch.zeros_like(val)
    for j in range(slot.shape[1]):
        rows = torch.nonzero(slot[:, j] >= 0).reshape(-1)
        at = slot[rows, j].long()
        tj = tf[rows]
        dy[at] = (tj * val[rows, j:j + 1]).to(dy.dtype)
        dval[rows, j] = (tj * y[at].float()).sum(dim=1)
    return dy, dval


def run(s):
    c = s["case"]
    op = c["op"]
    if not own:
        if op == "route_fwd":
            return _plain_route(c, s["logits"], s["bias"])
        if op == "route_vjp":
            return _plain_route_vjp(c, s["logits"], s["idx"], s["t"])
        if op == "map":
            return _places(s["idx"], c["n"], c["capacity"])
        if op == "product_fwd":
            return _plain_product(c, s["x"], s["w"], s["offset"], s["source"])
        if op == "product_vjp":
            return _plain_product_vjp(c, s["x"], s["w"], s["offset"], s["source"], s["t"])
        if op == "combine_fwd":
            return _plain_combine(s["y"], s["slot"], s["val"])
        return _plain_combine_vjp(s["y"], s["slot"], s["val"], s["t"], s["dy"])
    b = _lib()
    if op.startswith("route"):
        score = b.TOPK_SCORE_SIGMOID if c["score"] == "sigmoid" else b.TOPK_SCORE_SOFTMAX
        if op == "route_fwd":
            return b.topk_route_fwd(s["logits"], c["k"], score, bias=s["bias"], groups=c["groups"],
                                    keep_groups=c["keep"], group_top=c["top"], renormalise=c["renorm"])
        return b.topk_route_vjp(s["logits"], s["idx"], s["t"], score, renormalise=c["renorm"])
    if op == "map":
        return b.topk_expert_map(s["idx"], c["n"], capacity=c["capacity"])
    if op.startswith("product"):
        source = s["source"] if c["gather"] else None
        if op == "product_fwd":
            return b.topk_expert_product_fwd(s["x"], s["w"], s["offset"], source=source, k=c["k"])
        return b.topk_expert_product_vjp(s["x"], s["w"], s["offset"], s["t"], source=source, k=c["k"])
    if op == "combine_fwd":
        return b.topk_combine_fwd(s["y"], s["slot"], s["val"])
    return b.topk_combine_vjp(s["y"], s["slot"], s["val"], s["t"], dy_out=s["dy"])


# ---- the definition in 64 bits --------------------------------------------------------------------------------------

def _exact_route(case, logits, bias):
    l = np.where(np.isnan(logits), -np.inf, logits)
    rows, n, k = case["rows"], case["n"], case["k"]
    with np.errstate(all="ignore"):
        if case["score"] == "sigmoid":
            s = np.where(l >= 0, 1 / (1 + np.exp(-l)), np.exp(l) / (1 + np.exp(l)))
        else:
            m = l.max(axis=1, keepdims=True)
            s = np.exp(l - np.where(np.isinf(m), 0.0, m))
            z = s.sum(axis=1, keepdims=True)
            s = s / np.where(z == 0, 1.0, z)
    c = l if bias is None else s + bias[None, :]
    gone = np.isneginf(l) if bias is None else np.isneginf(l) | ~(bias > -np.inf)[None, :]
    c = np.where(gone, -np.inf, c)
    if case["groups"] > 1:
        summed = c if bias is not None or case["top"] == 1 else np.where(gone, -np.inf, s)
        part = -np.sort(-summed.reshape(rows, case["groups"], -1), axis=2)
        score = part[:, :, 0].copy()
        if case["top"] == 2 and part.shape[2] > 1:
            score += np.where(np.isneginf(part[:, :, 1]), 0.0, part[:, :, 1])
        place = np.argsort(np.argsort(-score, axis=1, kind="stable"), axis=1, kind="stable")
        c = np.where(np.repeat(place < case["keep"], n // case["groups"], axis=1), c, -np.inf)
    idx = np.argsort(-c, axis=1, kind="stable")[:, :k]
    empty = np.isneginf(np.take_along_axis(c, idx, axis=1))
    val = np.where(empty, 0.0, np.take_along_axis(s, idx, axis=1))
    if case["renorm"]:
        z = val.sum(axis=1, keepdims=True)
        val = val / np.where(z == 0, 1.0, z)
    return np.where(empty, -1, idx).astype(np.int32), val, s


def exact(case, seed):
    op, k = case["op"], case["k"]
    s = prepare(case, seed)
    if op.startswith("route"):
        logits = s["logits"].double().cpu().numpy()
        bias = None if s["bias"] is None else s["bias"].double().cpu().numpy()
        idx, val, score = _exact_route(case, logits, bias)
        if op == "route_fwd":
            return idx, val
        # the Jacobian's rows written out for the chosen entries
        idx = s["idx"].cpu().numpy()
        t = s["t"].double().cpu().numpy()
        at = np.where(idx < 0, 0, idx)
        there = idx >= 0
        p = np.where(there, np.take_along_axis(score, at, axis=1), 0.0)
        w = p
        if case["renorm"]:
            z = p.sum(axis=1, keepdims=True)
            w = p / np.where(z == 0, 1.0, z)
        mean = (t * w).sum(axis=1, keepdims=True)
        grad = np.zeros_like(score)
        r = np.arange(grad.shape[0])[:, None]
        if case["score"] == "softmax":
            if case["renorm"]:
                np.add.at(grad, (r, at), np.where(there, w * (t - mean), 0.0))
            else:
                np.add.at(grad, (r, at), np.where(there, w * t, 0.0))
                grad -= score * mean
        else:
            d = (w * (1 - p)) * ((t - mean) if case["renorm"] else t)
            np.add.at(grad, (r, at), np.where(there, d, 0.0))
        return grad
    if op == "map":
        idx = s["idx"].cpu().numpy()
        flat, n = idx.reshape(-1), case["n"]
        load = np.array([(flat == e).sum() for e in range(n)])
        most = case["capacity"] if case["capacity"] > 0 else flat.size
        offset = np.concatenate(([0], np.cumsum(np.minimum(load, most))))
        slot, source = np.full(flat.size, -1), np.full(flat.size, -1)
        for e in range(n):
            mine = np.flatnonzero(flat == e)[:most]
            slot[mine] = offset[e] + np.arange(mine.size)
            source[offset[e]:offset[e] + mine.size] = mine
        return tuple(a.astype(np.int32) for a in (slot.reshape(idx.shape), source, offset, load))
    if op.startswith("combine"):
        y, slot, val = s["y"].double(), s["slot"].long(), s["val"].double()
        rows, h = case["rows"], case["h"]
        at = slot.reshape(-1)
        there = at >= 0
        pair = torch.nonzero(there).reshape(-1)
        if op == "combine_fwd":
            out = torch.zeros((rows, h), dtype=torch.float64, device="cuda")
            return out.index_add_(0, pair // k, y[at[pair]] * val.reshape(-1, 1)[pair])
        t = s["t"].double()
        dy, dval = torch.zeros_like(y), torch.zeros_like(val)
        dy.index_copy_(0, at[pair], t[pair // k] * val.reshape(-1, 1)[pair])
        dval.view(-1)[pair] = (t[pair // k] * y[at[pair]]).sum(dim=1)
        return dy, dval
    at = s["offset"].cpu().numpy()
    x, w = s["x"], s["w"]
    pairs = case["rows"] * k
    row = s["source"].long() // k if case["gather"] else torch.arange(pairs, device="cuda")
    width = case["ho"] if op == "product_fwd" else case["h"]
    first = torch.zeros((pairs, width), dtype=torch.float64, device="cuda")
    dw = torch.zeros(w.shape, dtype=torch.float64, device="cuda") if op == "product_vjp" else None
    for e in np.flatnonzero(np.diff(at)):
        part = slice(int(at[e]), int(at[e + 1]))
        xe, we = x[row[part]].double(), w[e].double()
        if op == "product_fwd":
            first[part] = torch.mm(xe, we.t().contiguous())
        else:
            te = s["t"][part].double()
            first[part] = torch.mm(te, we)
            dw[e] = torch.mm(te.t().contiguous(), xe)
    return first if dw is None else (first, dw)


def work(case):
    """Bytes: every input read once, every output written once (of the experts' weights those that have rows, as many as
    independent choices would hit).  Operations: those of the products, elsewhere a handful per element."""
    op, rows, n, k = case["op"], case["rows"], case["n"], case["k"]
    pairs = rows * k
    if op.startswith("route"):
        e = _BYTES[case["dtype"]] * rows * n
        if op == "route_fwd":
            return {"bytes": float(e + 8 * pairs + (4 * n if case["bias"] else 0)), "flops": 6.0 * rows * n}
        # with softmax weights renormalised over the chosen only their logits enter, and so with sigmoid scores
        read = _BYTES[case["dtype"]] * pairs if case["renorm"] or case["score"] == "sigmoid" else e
        return {"bytes": float(read + 8 * pairs + e), "flops": 8.0 * rows * n}
    if op == "map":
        return {"bytes": float(12 * pairs + 4 * (2 * n + 1)), "flops": 2.0 * pairs}
    b = _BYTES[case["dtype"]]
    if op.startswith("combine"):
        rows_read = (1 if op == "combine_fwd" else 2) * pairs + rows
        return {"bytes": float(rows_read * case["h"] * b + pairs * (8 if op == "combine_fwd" else 12)),
                "flops": 2.0 * pairs * case["h"] * (1 if op == "combine_fwd" else 2)}
    h, ho = case["h"], case["ho"]
    hit = n * (1.0 - (1.0 - 1.0 / n) ** pairs)
    x = (rows if case["gather"] else pairs) * h
    lists = 4 * (n + 1) + (4 * pairs if case["gather"] else 0)
    if op == "product_fwd":
        return {"bytes": b * (x + hit * h * ho + pairs * ho) + lists, "flops": 2.0 * pairs * h * ho}
    return {"bytes": b * (x + pairs * ho + hit * h * ho + n * h * ho + pairs * h) + lists, "flops": 4.0 * pairs * h * ho}
