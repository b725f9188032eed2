"""The operators of a mixture of experts, as cases that can be timed: the router, the products grouped by expert, the
same products with 4-bit weights, and the weighted sum that brings the experts' rows back to their tokens.

`listed()` names the cases; `draw(rng)` gives further ones of the same ranges.  `run` computes a case in its plain form
(elementary torch operations in 32 bits, rounded once at the end) or, where `own` is true, through the library.

Words: a router gives each of T tokens `k` of E experts, which makes R = T * k pairs; the pairs are grouped by expert, in
the order of their tokens within one, and `order[r]` is the pair t * k + j that row r of that order stands for.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}


# --------------------------------------------------------------------------
# cases
# --------------------------------------------------------------------------

def _route(tokens, experts, k, dtype, renormalise, masked, grad):
    return {"op": "route", "tokens": tokens, "experts": experts, "k": k, "dtype": dtype, "renormalise": renormalise,
            "masked": masked, "grad": grad}


def _combine(tokens, k, width, dtype, grad):
    return {"op": "combine", "tokens": tokens, "k": k, "width": width, "dtype": dtype, "grad": grad}


def _mm(groups, tokens, k, inner, outer, dtype, layout, grad):
    """`k` > 0: the rows are gathered from `tokens` rows by a router's order; 0: they lie in order already."""
    return {"op": "mm", "groups": groups, "tokens": tokens, "k": k, "inner": inner, "outer": outer, "dtype": dtype,
            "layout": layout, "grad": grad}


def _w4(groups, tokens, k, inner, outer, dtype, group_k, zeros):
    """`group_k`: weights along the inner dimension that share a scale (and a zero point)."""
    return {"op": "w4", "groups": groups, "tokens": tokens, "k": k, "inner": inner, "outer": outer, "dtype": dtype,
            "group_k": group_k, "zeros": zeros}


def listed():
    named = {
        # one step of serving: a handful of tokens choose their experts; the call is all latency
        "route_4_tokens": _route(4, 64, 4, "f32", True, False, False),
        # the router of a training step, with the gradient of its logits
        "route_16k_train": _route(16_384, 128, 8, "bf16", True, False, True),
        # experts that some tokens may not use (a capacity rule, a device that is left out), whole rows masked, the
        # plain softmax as gates; sizes that nothing divides
        "route_masked_odd": _route(5_003, 60, 6, "f32", False, True, True),
        # the experts' rows summed up again while serving a few tokens, odd width
        "combine_13_tokens": _combine(13, 2, 1_001, "f16", False),
        # the same in a training step, with both gradients
        "combine_train": _combine(8_192, 4, 2_048, "bf16", True),
        # experts in 16 bits while serving: 16 tokens, two experts each; every weight in use is read for one or a few rows
        "mm_serve": _mm(16, 16, 2, 2_048, 4_096, "bf16", "nk", False),
        # a training step of the experts' first product, rows gathered by the router's order, with both gradients: the largest
        "mm_train": _mm(16, 8_192, 2, 2_048, 4_096, "bf16", "nk", True),
        # sizes that nothing divides, few groups of very different lengths, the other layout of the weights, both gradients
        "mm_odd_train": _mm(7, 3_001, 0, 1_000, 1_531, "f16", "kn", True),
        # the library's own type
        "mm_f32_train": _mm(8, 4_096, 0, 1_024, 1_024, "f32", "nk", True),
        # one token through one dense layer held in 4 bits
        "w4_one_token": _w4(1, 1, 0, 4_096, 4_096, "bf16", 128, False),
        # 16 tokens through four of 64 experts each: nearly every expert is read, for a row or two
        "w4_serve": _w4(64, 16, 4, 2_048, 1_408, "f16", 64, True),
        # a batch of requests through a large dense layer with fine scales
        "w4_batch": _w4(1, 48, 0, 8_192, 8_192, "bf16", 32, False),
    }
    return [{"name": name, **case} for name, case in named.items()]


def _log(rng, lo, hi):
    return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def _length(rng, lo, hi):
    """A power of two, an odd number or eight times an odd number."""
    v = _log(rng, lo, hi)
    kind = rng.randrange(3)
    if kind == 0:
        v = 1 << round(math.log2(v))
    elif kind == 1:
        v |= 1
    else:
        v = 8 * ((v // 8) | 1)
    return min(hi, max(lo, v))


def draw(rng):
    op = rng.choice(("route", "combine", "mm", "mm", "w4", "w4"))
    if op == "route":
        experts = _log(rng, 2, 512)
        return _route(_log(rng, 1, 32_768), experts, _log(rng, 1, min(16, experts)), rng.choice(("f32", "f16", "bf16")),
                      rng.random() < 0.5, rng.random() < 0.3, rng.random() < 0.5)
    if op == "combine":
        return _combine(_log(rng, 1, 16_384), rng.randint(1, 8), _length(rng, 64, 4_096), rng.choice(("f32", "f16", "bf16")),
                        rng.random() < 0.5)
    if op == "mm":
        most = 2 * 16_384 * 2_048 * 4_096
        while True:
            groups = _log(rng, 1, 64)
            k = rng.randint(0, min(8, groups))
            case = _mm(groups, _log(rng, 1, 8_192), k, _length(rng, 64, 4_096), _length(rng, 64, 4_096),
                       rng.choice(("f32", "f16", "bf16", "bf16")), rng.choice(("nk", "kn")), rng.random() < 0.5)
            flops = 2 * case["tokens"] * max(k, 1) * case["inner"] * case["outer"]
            if flops * (16 if case["dtype"] == "f32" else 1) <= most and groups * case["inner"] * case["outer"] <= 1 << 28:
                return case
    while True:
        groups = _log(rng, 1, 64)
        group_k = rng.choice((32, 64, 128))
        scales = _log(rng, 1, 8_192 // group_k)
        scales = 1 << round(math.log2(scales)) if rng.random() < 0.5 else min(scales | 1, 8_192 // group_k)
        case = _w4(groups, _log(rng, 1, 128), rng.randint(0, min(8, groups)), scales * group_k, _length(rng, 64, 8_192),
                   rng.choice(("f16", "bf16")), group_k, rng.random() < 0.5)
        if groups * case["inner"] * case["outer"] <= 1 << 28:
            return case


# --------------------------------------------------------------------------
# inputs
# --------------------------------------------------------------------------

def _normal(gen, *shape, scale=1.0, dtype=torch.float32):
    return (torch.randn(shape, generator=gen, device="cuda") * scale).to(dtype)


def _grouping(case, seed):
    """(bounds, order): where each group's rows begin and end, and the pair of each row (None where the rows lie in order).
    Some experts are chosen far more often than others, and some not at all."""
    rng = np.random.default_rng(seed)
    groups, tokens, k = case["groups"], case["tokens"], case["k"]
    liking = rng.normal(size=groups).astype(np.float32)
    if k == 0:
        share = np.exp(0.5 * liking)
        sizes = rng.multinomial(tokens, share / share.sum())
        return np.concatenate([[0], np.cumsum(sizes)]), None
    scores = 0.5 * liking + rng.gumbel(size=(tokens, groups)).astype(np.float32)
    experts = np.argpartition(-scores, k - 1, axis=1)[:, :k].reshape(-1)
    order = np.argsort(experts, kind="stable")
    return np.concatenate([[0], np.cumsum(np.bincount(experts, minlength=groups))]), order


def _prepare_route(case, gen, s):
    tokens, experts, k, dtype = case["tokens"], case["experts"], case["k"], TYPES[case["dtype"]]
    logits = _normal(gen, tokens, experts, scale=2.0, dtype=dtype)
    if case["masked"]:
        hidden = torch.rand((tokens, experts), generator=gen, device="cuda") < 0.3
        logits[hidden] = float("-inf")
        logits[1::89, 1:] = float("-inf")                # a row with one expert at most
        logits[2::97] = float("-inf")                    # a row with none
        logits[3::101] = torch.finfo(dtype).min          # a row masked with the lowest value: all of its experts alike
    s["logits"] = logits
    s["dgates"] = _normal(gen, tokens, k)
    if own:
        pairs = tokens * k
        s["gates"] = torch.empty((tokens, k), device="cuda")
        s["experts"], s["slot"] = (torch.empty((tokens, k), dtype=torch.int32, device="cuda") for _ in range(2))
        s["order"] = torch.empty(pairs, dtype=torch.int32, device="cuda")
        s["offsets"] = torch.empty(experts + 1, dtype=torch.int32, device="cuda")
        s["dlogits"] = torch.empty_like(logits)
        size = s["lib"].sgap_route_topk_workspace_size(tokens, experts, k)
        s["workspace"] = torch.empty(size, dtype=torch.uint8, device="cuda")


def _prepare_combine(case, gen, s, seed):
    tokens, k, width, dtype = case["tokens"], case["k"], case["width"], TYPES[case["dtype"]]
    rng = np.random.default_rng(seed)
    # rows of one expert lie in the order of their tokens; which experts a token has is drawn
    experts = np.argsort(rng.random((tokens, max(2 * k, 8))), axis=1)[:, :k].reshape(-1)
    order = np.argsort(experts, kind="stable")
    slot = np.empty(tokens * k, dtype=np.int64)
    slot[order] = np.arange(tokens * k)
    s["slot"] = torch.from_numpy(slot.astype(np.int32)).cuda().view(tokens, k)
    s["order"] = torch.from_numpy(order.astype(np.int32)).cuda()
    s["Z"] = _normal(gen, tokens * k, width, dtype=dtype)
    s["gates"] = torch.softmax(_normal(gen, tokens, k), dim=1)
    s["dout"] = _normal(gen, tokens, width, dtype=dtype)
    if own:
        s["out"] = torch.empty((tokens, width), dtype=dtype, device="cuda")
        s["dZ"] = torch.empty_like(s["Z"])
        s["dgates"] = torch.empty((tokens, k), device="cuda")


def _prepare_rows(case, gen, s, seed):
    """What both products have: the groups and the rows that come in."""
    bounds, order = _grouping(case, seed)
    s["bounds"] = bounds.tolist()
    s["offsets"] = torch.from_numpy(bounds.astype(np.int32)).cuda()
    s["src"] = None if order is None else torch.from_numpy(order.astype(np.int32)).cuda()
    s["rows"] = int(bounds[-1])
    s["X"] = _normal(gen, case["tokens"], case["inner"], dtype=TYPES[case["dtype"]])


def _prepare_mm(case, gen, s, seed):
    groups, inner, outer, dtype = case["groups"], case["inner"], case["outer"], TYPES[case["dtype"]]
    _prepare_rows(case, gen, s, seed)
    shape = (groups, outer, inner) if case["layout"] == "nk" else (groups, inner, outer)
    s["W"] = _normal(gen, *shape, scale=inner ** -0.5, dtype=dtype)
    if case["grad"]:
        s["dY"] = _normal(gen, s["rows"], outer, dtype=dtype)
    if own:
        s["Y"] = torch.empty((s["rows"], outer), dtype=dtype, device="cuda")
        if case["grad"]:
            s["dX"] = torch.empty((s["rows"], inner), dtype=dtype, device="cuda")
            s["dW"] = torch.empty_like(s["W"])


def _prepare_w4(case, gen, s, seed):
    groups, inner, outer, dtype = case["groups"], case["inner"], case["outer"], TYPES[case["dtype"]]
    _prepare_rows(case, gen, s, seed)
    blocks = inner // case["group_k"]
    # a quantised weight: normally distributed codes, the even one of two neighbours in a byte's low half
    quant = torch.empty((groups, outer, inner // 2), dtype=torch.uint8, device="cuda")
    for g in range(groups):
        codes = (_normal(gen, outer, inner, scale=2.6) + 8.0).round_().clamp_(0, 15).to(torch.uint8)
        quant[g] = codes[:, 0::2] | (codes[:, 1::2] << 4)
    s["quant"] = quant
    s["scales"] = ((0.5 + torch.rand((groups, outer, blocks), generator=gen, device="cuda")) * (0.4 * inner ** -0.5)).to(dtype)
    s["zeros"] = None
    if case["zeros"]:
        s["zeros"] = torch.randint(5, 12, (groups, outer, blocks), generator=gen, device="cuda").to(torch.uint8)
    if own:
        # the weights as the library keeps them: laid out once when they are loaded
        lib = s["lib"]
        size = lib.sgap_w4_layout_size(groups, inner, outer, case["group_k"], zeros=case["zeros"])
        s["weights"] = torch.empty(size, dtype=torch.uint8, device="cuda")
        lib.sgap_w4_layout(groups, inner, outer, case["group_k"], quant, s["scales"], s["zeros"], s["weights"])
        s["Y"] = torch.empty((s["rows"], outer), dtype=dtype, device="cuda")


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    s = {"case": case}
    if own:
        from paper_2209_02882_amd import binding

        s["lib"] = binding
    if case["op"] == "route":
        _prepare_route(case, gen, s)
    elif case["op"] == "combine":
        _prepare_combine(case, gen, s, seed)
    elif case["op"] == "mm":
        _prepare_mm(case, gen, s, seed)
    else:
        _prepare_w4(case, gen, s, seed)
    return s


# --------------------------------------------------------------------------
# one pass
# --------------------------------------------------------------------------

def _plain_route(s, case):
    logits, k = s["logits"], case["k"]
    experts_of = case["experts"]
    x = logits.float()
    # stable and descending: equal logits in the order of their experts
    top, experts = torch.sort(x, dim=1, descending=True, stable=True)
    top, experts = top[:, :k], experts[:, :k]
    there = top > float("-inf")
    most = torch.where(there[:, :1], top[:, :1], torch.zeros_like(top[:, :1]))
    e = torch.exp(x - most)
    chosen_e = torch.exp(top - most)
    total = (chosen_e if case["renormalise"] else e).sum(dim=1, keepdim=True)
    total = torch.where(total > 0, total, torch.ones_like(total))
    gates = chosen_e / total
    experts = torch.where(there, experts, torch.full_like(experts, experts_of))  # behind every expert
    flat = experts.reshape(-1)
    order = torch.sort(flat, stable=True)[1]
    ranks = torch.arange(flat.numel(), device=flat.device)
    slot = torch.empty_like(order)
    slot[order] = ranks
    counts = torch.zeros(experts_of + 1, dtype=torch.int64, device=flat.device)
    counts.index_add_(0, flat, torch.ones_like(flat))
    offsets = torch.zeros(experts_of + 1, dtype=torch.int64, device=flat.device)
    offsets[1:] = torch.cumsum(counts[:-1], 0)
    used = offsets[-1]
    order = torch.where(ranks < used, order, torch.full_like(order, -1))
    slot = torch.where(there, slot.view_as(experts), torch.full_like(experts, -1))
    experts_out = torch.where(there, experts, torch.full_like(experts, -1))
    out = [gates, experts_out.int(), slot.int(), order.int(), offsets.int()]
    if case["grad"]:
        inner = (gates * s["dgates"]).sum(dim=1, keepdim=True)
        if case["renormalise"]:
            dl = torch.zeros_like(x)
            part = torch.where(there, gates * (s["dgates"] - inner), torch.zeros_like(gates))
        else:
            dl = -(e / total) * inner
            part = gates * s["dgates"]
        dl.scatter_add_(1, torch.where(there, experts, torch.zeros_like(experts)), part)
        out.append(dl.to(logits.dtype))
    return out


def _plain_combine(s, case):
    z = s["Z"][s["slot"].long().reshape(-1)].view(case["tokens"], case["k"], -1).float()
    out = [(z * s["gates"].unsqueeze(2)).sum(dim=1).to(s["Z"].dtype)]
    if case["grad"]:
        d = s["dout"].float()
        out.append((d[(s["order"] // case["k"]).long()] * s["gates"].reshape(-1)[s["order"].long()].unsqueeze(1)).to(s["Z"].dtype))
        out.append((z * d.unsqueeze(1)).sum(dim=2))
    return out


def _plain_rows(s, case, a, b):
    if s["src"] is None:
        return s["X"][a:b].float()
    return s["X"][(s["src"][a:b] // case["k"]).long()].float()


def _plain_mm(s, case):
    nk = case["layout"] == "nk"
    W = s["W"]
    Y = torch.empty((s["rows"], case["outer"]), dtype=W.dtype, device="cuda")
    if case["grad"]:
        dX = torch.empty((s["rows"], case["inner"]), dtype=W.dtype, device="cuda")
        dW = torch.zeros_like(W)
    for g in range(case["groups"]):
        a, b = s["bounds"][g], s["bounds"][g + 1]
        if a == b:
            continue
        x, w = _plain_rows(s, case, a, b), W[g].float()
        Y[a:b] = x @ (w.t() if nk else w)
        if case["grad"]:
            d = s["dY"][a:b].float()
            dX[a:b] = d @ (w if nk else w.t())
            dW[g] = d.t() @ x if nk else x.t() @ d
    return [Y, dX, dW] if case["grad"] else [Y]


def _plain_w4(s, case):
    Y = torch.empty((s["rows"], case["outer"]), dtype=s["X"].dtype, device="cuda")
    for g in range(case["groups"]):
        a, b = s["bounds"][g], s["bounds"][g + 1]
        if a == b:
            continue
        q = s["quant"][g]
        w = torch.stack([q & 15, q >> 4], dim=2).float().view(case["outer"], -1, case["group_k"])
        zero = 8.0 if s["zeros"] is None else s["zeros"][g].float().unsqueeze(2)
        w = ((w - zero) * s["scales"][g].float().unsqueeze(2)).view(case["outer"], case["inner"])
        Y[a:b] = _plain_rows(s, case, a, b) @ w.t()
    return [Y]


def run(s):
    case = s["case"]
    op = case["op"]
    if not own:
        return {"route": _plain_route, "combine": _plain_combine, "mm": _plain_mm, "w4": _plain_w4}[op](s, case)
    lib = s["lib"]
    if op == "route":
        tokens, experts, k = case["tokens"], case["experts"], case["k"]
        lib.sgap_route_topk(tokens, experts, k, s["logits"], s["gates"], s["experts"], s["slot"], s["order"], s["offsets"],
                            renormalise=case["renormalise"], workspace=s["workspace"])
        out = [s["gates"], s["experts"], s["slot"], s["order"], s["offsets"]]
        if case["grad"]:
            lib.sgap_route_topk_grad(tokens, experts, k, s["logits"], s["gates"], s["experts"], s["dgates"], s["dlogits"],
                                     renormalise=case["renormalise"])
            out.append(s["dlogits"])
        return out
    if op == "combine":
        tokens, k, width = case["tokens"], case["k"], case["width"]
        lib.sgap_route_combine(tokens, k, width, s["Z"], s["slot"], s["gates"], s["out"])
        if not case["grad"]:
            return [s["out"]]
        lib.sgap_route_combine_grad(tokens, k, width, s["Z"], s["slot"], s["order"], s["gates"], s["dout"], s["dZ"], s["dgates"])
        return [s["out"], s["dZ"], s["dgates"]]
    groups, inner, outer, rows = case["groups"], case["inner"], case["outer"], s["rows"]
    gather = {} if s["src"] is None else {"src": s["src"], "src_div": case["k"]}
    if op == "w4":
        lib.sgap_grouped_mm_w4(groups, rows, inner, outer, case["group_k"], s["offsets"], s["X"], s["weights"], s["Y"],
                               zeros=case["zeros"], **gather)
        return [s["Y"]]
    layout = case["layout"]
    lib.sgap_grouped_mm(groups, rows, inner, outer, s["offsets"], s["X"], s["W"], s["Y"], layout, **gather)
    if not case["grad"]:
        return [s["Y"]]
    lib.sgap_grouped_mm(groups, rows, outer, inner, s["offsets"], s["dY"], s["W"], s["dX"], "kn" if layout == "nk" else "nk")
    lib.sgap_grouped_mm_wgrad(groups, rows, inner, outer, s["offsets"], s["X"], s["dY"], s["dW"], layout, **gather)
    return [s["Y"], s["dX"], s["dW"]]


# --------------------------------------------------------------------------
# the definition in 64 bits
# --------------------------------------------------------------------------

def _exact_route(s, case):
    x = s["logits"].double().cpu().numpy()
    tokens, experts_of, k = case["tokens"], case["experts"], case["k"]
    dg = s["dgates"].double().cpu().numpy()
    chosen = np.argsort(-x, axis=1, kind="stable")[:, :k]
    rows = np.arange(tokens)[:, None]
    there = np.isfinite(x[rows, chosen])
    p = np.zeros_like(x)
    some = np.isfinite(x).any(axis=1)
    p[some] = np.exp(x[some] - x[some].max(axis=1, keepdims=True))
    p[some] /= p[some].sum(axis=1, keepdims=True)
    gates = np.where(there, p[rows, chosen], 0.0)
    if case["renormalise"]:
        total = gates.sum(axis=1, keepdims=True)
        gates = gates / np.where(total > 0, total, 1.0)
    pairs = [(int(e), i) for i, e in enumerate(np.where(there, chosen, -1).reshape(-1)) if e >= 0]
    pairs.sort()
    order = np.full(tokens * k, -1, dtype=np.int32)
    slot = np.full(tokens * k, -1, dtype=np.int32)
    order[:len(pairs)] = [i for _, i in pairs]
    slot[order[:len(pairs)]] = np.arange(len(pairs))
    offsets = np.searchsorted(np.array([e for e, _ in pairs], dtype=np.int64), np.arange(experts_of + 1)).astype(np.int32)
    out = [torch.from_numpy(gates), torch.from_numpy(np.where(there, chosen, -1).astype(np.int32)),
           torch.from_numpy(slot.reshape(tokens, k)), torch.from_numpy(order), torch.from_numpy(offsets)]
    if case["grad"]:
        # the Jacobian of the gates, one chosen expert after the other
        dl = np.zeros_like(x)
        dense = np.zeros_like(x)
        np.put_along_axis(dense, chosen, np.where(there, gates, 0.0), axis=1)
        base = dense if case["renormalise"] else p
        for j in range(k):
            w = np.where(there[:, j], gates[:, j] * dg[:, j], 0.0)
            dl -= w[:, None] * base
            dl[np.arange(tokens), chosen[:, j]] += w
        out.append(torch.from_numpy(dl))
    return out


def _exact_combine(s, case):
    tokens, k = case["tokens"], case["k"]
    Z, gates, slot = s["Z"].double(), s["gates"].double(), s["slot"].long()
    out = torch.zeros((tokens, case["width"]), dtype=torch.float64, device="cuda")
    for j in range(k):
        out += Z[slot[:, j]] * gates[:, j:j + 1]
    if not case["grad"]:
        return [out]
    d = s["dout"].double()
    dZ, dg = torch.zeros_like(Z), torch.zeros_like(gates)
    for j in range(k):
        dZ[slot[:, j]] = gates[:, j:j + 1] * d
        dg[:, j] = (Z[slot[:, j]] * d).sum(dim=1)
    return [out, dZ, dg]


def _exact_products(s, case, weight):
    """`weight(g)`: the group's weights in 64 bits, outer x inner."""
    rows = torch.arange(s["rows"], device="cuda") if s["src"] is None else torch.div(s["src"].long(), case["k"], rounding_mode="floor")
    X = s["X"].double()[rows]
    Y = torch.zeros((s["rows"], case["outer"]), dtype=torch.float64, device="cuda")
    grad = case.get("grad", False)
    if grad:
        D = s["dY"].double()
        dX = torch.zeros((s["rows"], case["inner"]), dtype=torch.float64, device="cuda")
        dW = torch.zeros(s["W"].shape, dtype=torch.float64, device="cuda")
    for g, (a, b) in enumerate(zip(s["bounds"], s["bounds"][1:])):
        if b > a:
            w = weight(g)
            Y[a:b] = torch.mm(X[a:b], w.t().contiguous())
            if grad:
                dX[a:b] = torch.mm(D[a:b], w)
                outer_inner = torch.mm(D[a:b].t().contiguous(), X[a:b])
                dW[g] = outer_inner if case["layout"] == "nk" else outer_inner.t()
    return [Y, dX, dW] if grad else [Y]


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "route":
        return _exact_route(s, case)
    if case["op"] == "combine":
        return _exact_combine(s, case)
    if case["op"] == "mm":
        return _exact_products(s, case, lambda g: (s["W"][g] if case["layout"] == "nk" else s["W"][g].t()).double().contiguous())

    def weight(g):
        q, n = s["quant"][g].to(torch.int64), case["group_k"]
        w = torch.empty((case["outer"], case["inner"]), dtype=torch.float64, device="cuda")
        w[:, 0::2], w[:, 1::2] = (q % 16).double(), torch.div(q, 16, rounding_mode="floor").double()
        zero = torch.full_like(s["scales"][g], 8).double() if s["zeros"] is None else s["zeros"][g].double()
        return (w - zero.repeat_interleave(n, dim=1)) * s["scales"][g].double().repeat_interleave(n, dim=1)

    return _exact_products(s, case, weight)


# --------------------------------------------------------------------------
# what a pass cannot do without
# --------------------------------------------------------------------------

def _groups_in_use(case):
    """Groups that have a row, in the mean over the draws of `_grouping` (alike groups taken for unlike ones)."""
    groups, k = case["groups"], case["k"]
    missed = (1 - k / groups) ** case["tokens"] if k else (1 - 1 / groups) ** case["tokens"]
    return groups * (1 - missed)


def work(case):
    size = BYTES[case["dtype"]]
    if case["op"] == "route":
        tokens, experts, k = case["tokens"], case["experts"], case["k"]
        moved = tokens * experts * size + tokens * k * 16 + (experts + 1) * 4
        if case["grad"]:
            moved += tokens * k * 4 + tokens * experts * size
        return {"bytes": moved, "flops": tokens * experts * (8 if case["grad"] else 4)}
    if case["op"] == "combine":
        tokens, k, width = case["tokens"], case["k"], case["width"]
        pairs = tokens * k
        moved = pairs * width * size + pairs * 8 + tokens * width * size
        if case["grad"]:
            moved += tokens * width * size + pairs * width * size + pairs * 8
        return {"bytes": moved, "flops": pairs * width * (5 if case["grad"] else 2)}
    rows, inner, outer, used = case["tokens"] * max(case["k"], 1), case["inner"], case["outer"], _groups_in_use(case)
    lists = (case["groups"] + 1) * 4 + (rows * 4 if case["k"] else 0)
    inputs = case["tokens"] * inner * size
    if case["op"] == "w4":
        weights = inner * outer / 2 + outer * (inner // case["group_k"]) * (size + (1 if case["zeros"] else 0))
        return {"bytes": lists + inputs + used * weights + rows * outer * size, "flops": 2 * rows * inner * outer}
    moved = lists + inputs + used * inner * outer * size + rows * outer * size
    if case["grad"]:
        moved += rows * outer * size + rows * inner * size + case["groups"] * inner * outer * size
    return {"bytes": moved, "flops": 2 * rows * inner * outer * (3 if case["grad"] else 1)}
