"""What a mixture of experts that is trained on tokens needs around its products, as cases that can be timed: the rows of
an embedding and their gradient, the router's balance loss with its counts and its gradient, numbers of 8 bits with a scale
for each block of 128, and the products of rows grouped by expert in them.

`listed()` names the cases; `draw(rng)` gives further ones of the same ranges.  `run` computes a case in its plain form
(elementary torch operations in 32 bits, rounded once at the end) or, where `own` is true, through the library.

Words: T tokens, a vocabulary of V rows; R rows of a product, grouped by expert; numbers of 8 bits are e4m3 (four bits of
exponent, three of mantissa, no infinity, largest 448), called codes, and a block's scale times a code is the value.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}
BLOCK = 128
LARGEST = 448.0


def _blocks(n):
    return (n + BLOCK - 1) // BLOCK


# --------------------------------------------------------------------------
# cases
# --------------------------------------------------------------------------

def _embed(tokens, vocabulary, width, dtype, scale, padding, steps, grad_dtype):
    """`steps`: batches whose gradients are summed up, the first overwriting, the others adding; 0: no gradient."""
    return {"op": "embed", "tokens": tokens, "vocabulary": vocabulary, "width": width, "dtype": dtype, "scale": scale,
            "padding": padding, "steps": steps, "grad_dtype": grad_dtype}


def _balance(tokens, experts, k, sequences, dtype, padding):
    return {"op": "balance", "tokens": tokens, "experts": experts, "k": k, "sequences": sequences, "dtype": dtype, "padding": padding}


def _weights(groups, inner, outer, dtype, both):
    """`both`: as they are and transposed, which the gradient of the rows wants."""
    return {"op": "weights", "groups": groups, "inner": inner, "outer": outer, "dtype": dtype, "both": both}


def _rows(rows, inner, dtype):
    return {"op": "rows", "rows": rows, "inner": inner, "dtype": dtype}


def _mm(groups, tokens, k, inner, outer, dtype, grad):
    """`k` > 0: the rows are gathered from `tokens` rows by a router's order; 0: they lie in order already."""
    return {"op": "mm", "groups": groups, "tokens": tokens, "k": k, "inner": inner, "outer": outer, "dtype": dtype, "grad": grad}


def listed():
    named = {
        # one step of serving: the rows of a few tokens out of a large vocabulary; the call is all latency
        "embed_8_tokens": _embed(8, 131_072, 4_096, "bf16", 1.0, False, 0, "bf16"),
        # a training step: the rows of a batch, and the gradient of the whole table, most of whose rows no token has
        "embed_train": _embed(16_384, 65_536, 2_048, "bf16", 1.0, False, 1, "bf16"),
        # two batches that add up in a gradient of floats, padded sequences, a scale, sizes that nothing divides
        "embed_padded_odd": _embed(5_003, 50_001, 1_001, "f16", 1_001 ** 0.5, True, 2, "f32"),
        # the loss that keeps the experts of a training step evenly used, over the whole batch
        "balance_train": _balance(16_384, 128, 8, 1, "bf16", False),
        # the same for each of a batch's packed sequences, of very different lengths, with padding behind them
        "balance_packed_odd": _balance(5_003, 60, 6, 37, "f32", True),
        # the experts' weights, which a training step puts into 8 bits again after each update, both ways round
        "f8_weights_train": _weights(16, 2_048, 4_096, "bf16", True),
        # rows that are put into 8 bits on their own, sizes that nothing divides
        "f8_rows_odd": _rows(3_001, 1_000, "f16"),
        # one token through one dense layer held in 8 bits: latency and the weights' bytes
        "f8_one_token": _mm(1, 1, 0, 4_096, 4_096, "bf16", False),
        # 16 tokens through four of 64 experts each: nearly every expert is read, for a row or two
        "f8_serve": _mm(64, 16, 4, 2_048, 1_408, "f16", False),
        # a prompt through a large dense layer
        "f8_prompt": _mm(1, 8_192, 0, 4_096, 8_192, "bf16", False),
        # a training step of the experts' first product, rows gathered by the router's order, with the gradient of the rows: the largest
        "f8_train": _mm(16, 8_192, 2, 2_048, 4_096, "bf16", True),
        # sizes that nothing divides, few groups of very different lengths, with the gradient of the rows
        "f8_odd_train": _mm(7, 3_001, 0, 1_000, 1_531, "f16", True),
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
    op = rng.choice(("embed", "balance", "weights", "rows", "mm", "mm"))
    dtype = rng.choice(("f32", "f16", "bf16"))
    if op == "embed":
        while True:
            case = _embed(_log(rng, 1, 32_768), _log(rng, 64, 262_144), _length(rng, 64, 8_192), dtype,
                          rng.choice((1.0, 0.5, 27.7)), rng.random() < 0.4, rng.choice((0, 1, 1, 2)), rng.choice((dtype, "f32")))
            if case["vocabulary"] * case["width"] <= 1 << 28 and case["tokens"] * case["width"] <= 1 << 26:
                return case
    if op == "balance":
        experts = _log(rng, 2, 512)
        tokens = _log(rng, 1, 65_536)
        return _balance(tokens, experts, _log(rng, 1, min(16, experts)), rng.choice((1, _log(rng, 1, 300))), dtype, rng.random() < 0.4)
    if op == "weights":
        while True:
            case = _weights(_log(rng, 1, 64), _length(rng, 64, 8_192), _length(rng, 64, 8_192), dtype, rng.random() < 0.5)
            if case["groups"] * case["inner"] * case["outer"] <= 1 << 28:
                return case
    if op == "rows":
        while True:
            case = _rows(_log(rng, 1, 32_768), _length(rng, 64, 16_384), dtype)
            if case["rows"] * case["inner"] <= 1 << 28:
                return case
    most = 2 * 8_192 * 4_096 * 8_192
    while True:
        groups = _log(rng, 1, 64)
        case = _mm(groups, _log(rng, 1, 8_192), rng.randint(0, min(8, groups)), _length(rng, 64, 8_192), _length(rng, 64, 8_192),
                   dtype, rng.random() < 0.5)
        flops = 2 * case["tokens"] * max(case["k"], 1) * case["inner"] * case["outer"] * (2 if case["grad"] else 1)
        if flops <= most and groups * case["inner"] * case["outer"] <= 1 << 28:
            return case


# --------------------------------------------------------------------------
# inputs
# --------------------------------------------------------------------------

def _normal(gen, *shape, scale=1.0, dtype=torch.float32):
    return (torch.randn(shape, generator=gen, device="cuda") * scale).to(dtype)


def _prepare_embed(case, gen, s):
    tokens, vocabulary, width, dtype = case["tokens"], case["vocabulary"], case["width"], TYPES[case["dtype"]]
    s["W"] = _normal(gen, vocabulary, width, scale=0.02, dtype=dtype)
    ids, dout = [], []
    for _ in range(max(case["steps"], 1)):
        # a token's frequency goes with one over its rank, the ranks lie anywhere in the table
        u = torch.rand(tokens, generator=gen, device="cuda", dtype=torch.float64)
        rank = torch.exp(u * math.log(vocabulary + 1)).long().clamp(1, vocabulary) - 1
        id_of = torch.randperm(vocabulary, generator=gen, device="cuda")
        these = id_of[rank].int()
        if case["padding"]:
            # sequences of 500 places, each filled to some part of it
            at = torch.arange(tokens, device="cuda")
            filled = torch.randint(1, 501, ((tokens + 499) // 500,), generator=gen, device="cuda")
            these = torch.where(at % 500 < filled[at // 500], these, torch.full_like(these, -1))
        ids.append(these)
        dout.append(_normal(gen, tokens, width, dtype=dtype))
    s["ids"], s["dout"] = ids, dout
    if own:
        s["out"] = [torch.empty((tokens, width), dtype=dtype, device="cuda") for _ in ids]
        if case["steps"]:
            s["dW"] = torch.empty((vocabulary, width), dtype=TYPES[case["grad_dtype"]], device="cuda")
            s["workspace"] = torch.empty(s["lib"].sgap_embed_grad_workspace_size(tokens, vocabulary, width), dtype=torch.uint8, device="cuda")


def _prepare_balance(case, gen, s, seed):
    tokens, experts, k, sequences, dtype = case["tokens"], case["experts"], case["k"], case["sequences"], TYPES[case["dtype"]]
    rng = np.random.default_rng(seed)
    # some experts are liked more than others
    logits = (_normal(gen, tokens, experts, scale=1.5) + _normal(gen, experts)).to(dtype)
    ends = np.sort(rng.integers(0, tokens + 1, size=sequences - 1)) if sequences > 1 else np.zeros(0, dtype=np.int64)
    last = tokens - tokens // 20 if case["padding"] else tokens
    bounds = np.concatenate([[0], np.minimum(ends, last), [last]])
    if case["padding"]:
        at = torch.arange(tokens, device="cuda")
        logits[(at % 11 == 3) | (at >= last)] = float("-inf")   # places without a token, between the sequences' tokens and behind them
        hidden = torch.rand((tokens, experts), generator=gen, device="cuda") < 0.2
        logits[hidden & (at % 2 == 0).unsqueeze(1)] = float("-inf")
    s["logits"], s["bounds"] = logits, bounds.tolist()
    s["segments"] = None if sequences == 1 and not case["padding"] else torch.from_numpy(bounds.astype(np.int32)).cuda()
    top, chosen = torch.sort(logits.float(), dim=1, descending=True, stable=True)
    s["experts"] = torch.where(top[:, :k] > float("-inf"), chosen[:, :k], torch.full_like(chosen[:, :k], -1)).int().contiguous()
    s["dloss"] = torch.full((1,), 0.01, device="cuda")
    if own:
        s["loss"] = torch.empty(1, device="cuda")
        s["counts"] = torch.empty((sequences, experts), dtype=torch.int32, device="cuda")
        s["rows"] = torch.empty(sequences, dtype=torch.int32, device="cuda")
        s["dlogits"] = torch.empty_like(logits)
        size = s["lib"].sgap_route_balance_workspace_size(tokens, experts, k, sequences)
        s["workspace"] = torch.empty(size, dtype=torch.uint8, device="cuda")


def _empty_codes(*shape):
    return torch.empty(shape, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)


def _prepare_weights(case, gen, s):
    groups, inner, outer, dtype = case["groups"], case["inner"], case["outer"], TYPES[case["dtype"]]
    # outputs of very different size, as trained weights have
    s["W"] = (_normal(gen, groups, outer, inner, scale=inner ** -0.5) * torch.exp(_normal(gen, groups, outer, 1))).to(dtype)
    if own:
        s["codes"] = _empty_codes(groups, outer, BLOCK * _blocks(inner))
        s["scales"] = torch.empty((groups, _blocks(outer), _blocks(inner)), device="cuda")
        s["codes_t"] = s["scales_t"] = None
        if case["both"]:
            s["codes_t"] = _empty_codes(groups, inner, BLOCK * _blocks(outer))
            s["scales_t"] = torch.empty((groups, _blocks(inner), _blocks(outer)), device="cuda")


def _prepare_rows(case, gen, s):
    rows, inner, dtype = case["rows"], case["inner"], TYPES[case["dtype"]]
    s["X"] = (_normal(gen, rows, inner) * torch.exp(_normal(gen, 1, inner))).to(dtype)   # some columns are far larger than others
    if own:
        s["codes"] = _empty_codes(rows, BLOCK * _blocks(inner))
        s["scales"] = torch.empty((rows, _blocks(inner)), device="cuda")


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


def _prepare_mm(case, gen, s, seed):
    groups, inner, outer, dtype = case["groups"], case["inner"], case["outer"], TYPES[case["dtype"]]
    bounds, order = _grouping(case, seed)
    s["bounds"], s["rows"] = bounds.tolist(), int(bounds[-1])
    s["offsets"] = torch.from_numpy(bounds.astype(np.int32)).cuda()
    s["src"] = None if order is None else torch.from_numpy(order.astype(np.int32)).cuda()
    s["X"] = _normal(gen, case["tokens"], inner, dtype=dtype)
    # weights as a checkpoint has them: codes in rows of whole blocks, zeros behind the last value, and any float as a scale
    nb, kb = _blocks(outer), _blocks(inner)
    codes = torch.zeros((groups, BLOCK * nb, BLOCK * kb), dtype=torch.uint8, device="cuda")
    s["w_scales"] = torch.empty((groups, nb, kb), device="cuda")
    for g in range(groups):
        w = torch.zeros((BLOCK * nb, BLOCK * kb), device="cuda")
        w[:outer, :inner] = _normal(gen, outer, inner, scale=inner ** -0.5) * torch.exp(0.5 * _normal(gen, outer, 1))
        t = w.view(nb, BLOCK, kb, BLOCK)
        scale = t.abs().amax(dim=(1, 3)) / LARGEST
        s["w_scales"][g] = scale
        codes[g] = (t / scale.view(nb, 1, kb, 1)).clamp(-LARGEST, LARGEST).view_as(w).to(torch.float8_e4m3fn).view(torch.uint8)
    s["w_codes"] = codes[:, :outer].contiguous().view(torch.float8_e4m3fn)
    if case["grad"]:
        s["dY"] = _normal(gen, s["rows"], outer, scale=1e-3, dtype=dtype)
    if own:
        s["x_codes"] = _empty_codes(case["tokens"], BLOCK * kb)
        s["x_scales"] = torch.empty((case["tokens"], kb), device="cuda")
        s["Y"] = torch.empty((s["rows"], outer), dtype=dtype, device="cuda")
        if case["grad"]:
            s["t_codes"] = codes.transpose(1, 2)[:, :inner].contiguous().view(torch.float8_e4m3fn)
            s["t_scales"] = s["w_scales"].transpose(1, 2).contiguous()
            s["d_codes"] = _empty_codes(s["rows"], BLOCK * nb)
            s["d_scales"] = torch.empty((s["rows"], nb), device="cuda")
            s["dX"] = torch.empty((s["rows"], inner), dtype=dtype, device="cuda")


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    s = {"case": case}
    if own:
        from paper_2209_02882_amd import binding

        s["lib"] = binding
    if case["op"] == "embed":
        _prepare_embed(case, gen, s)
    elif case["op"] == "balance":
        _prepare_balance(case, gen, s, seed)
    elif case["op"] == "weights":
        _prepare_weights(case, gen, s)
    elif case["op"] == "rows":
        _prepare_rows(case, gen, s)
    else:
        _prepare_mm(case, gen, s, seed)
    return s


# --------------------------------------------------------------------------
# one pass
# --------------------------------------------------------------------------

def _plain_embed(s, case):
    out = []
    for ids in s["ids"]:
        there = ids >= 0
        rows = s["W"][torch.where(there, ids, torch.zeros_like(ids)).long()].float() * case["scale"]
        out.append((rows * there.unsqueeze(1)).to(s["W"].dtype))
    if not case["steps"]:
        return out
    dW = torch.zeros((case["vocabulary"] + 1, case["width"]), device="cuda")
    for ids, dout in zip(s["ids"], s["dout"]):
        dW.index_add_(0, torch.where(ids >= 0, ids, torch.full_like(ids, case["vocabulary"])).long(), dout.float() * case["scale"])
    return out + [dW[:case["vocabulary"]].to(TYPES[case["grad_dtype"]])]


def _plain_balance(s, case):
    tokens, experts, k, sequences = case["tokens"], case["experts"], case["k"], case["sequences"]
    x = s["logits"].float()
    there = s["experts"][:, :1] >= 0
    if s["segments"] is None:
        which = torch.zeros(tokens, dtype=torch.int64, device="cuda")
    else:
        which = torch.searchsorted(s["segments"], torch.arange(tokens, dtype=torch.int32, device="cuda"), right=True).long() - 1
    which = torch.where(there[:, 0], which, torch.full_like(which, sequences))   # places without a token: a sequence of their own
    most = torch.where(there, x.amax(dim=1, keepdim=True), torch.zeros_like(x[:, :1]))
    p = torch.exp(x - most)
    p = p / torch.where(there, p.sum(dim=1, keepdim=True), torch.ones_like(most))
    rows = torch.zeros(sequences + 1, dtype=torch.int64, device="cuda").index_add_(0, which, torch.ones_like(which))[:sequences]
    chosen = torch.where(s["experts"] >= 0, which.unsqueeze(1) * experts + s["experts"], torch.full_like(which, sequences * experts).unsqueeze(1))
    counts = torch.zeros(sequences * experts + 1, dtype=torch.int64, device="cuda")
    counts = counts.index_add_(0, chosen.reshape(-1), torch.ones_like(chosen.reshape(-1)))[:-1].view(sequences, experts)
    n = rows.clamp(min=1).float().unsqueeze(1)
    used = (rows > 0).sum().clamp(min=1).float()
    share = torch.zeros((sequences + 1, experts), device="cuda").index_add_(0, which, p)[:sequences] / n
    # the shares of the experts less one, as whole numbers until they are divided: where all are alike, nothing is left
    f = (counts * experts - k * rows.unsqueeze(1)).float() / (k * n)
    loss = ((f + 1) * share).sum() / used
    scale = torch.cat([s["dloss"] / (used * n[:, 0]), torch.zeros(1, device="cuda")])
    f = torch.cat([f, torch.zeros((1, experts), device="cuda")])[which]
    dlogits = scale[which].unsqueeze(1) * p * (f - (f * p).sum(dim=1, keepdim=True))
    return [loss.view(1), counts.int(), rows.int(), dlogits.to(s["logits"].dtype)]


def _power_scales(most):
    """The smallest power of two, 2^-126 at least, that times the largest code is `most` or more; 1 where there is nothing."""
    mantissa, exponent = torch.frexp(most.double() / LARGEST)
    exponent = (exponent - (mantissa == 0.5).to(exponent.dtype)).clamp(min=-126)
    # a float's bits, its exponent in the place of bits 23 to 30
    return torch.where(most > 0, (exponent + 127 << 23).to(torch.int32).view(torch.float32), torch.ones_like(most, dtype=torch.float32))


def _plain_rows(x):
    """(codes, in rows of whole blocks, and scales) of the rows of x."""
    rows, inner = x.shape
    kb = _blocks(inner)
    whole = torch.zeros((rows, BLOCK * kb), device="cuda")
    whole[:, :inner] = x.float()
    t = whole.view(rows, kb, BLOCK)
    scales = _power_scales(t.abs().amax(dim=2))
    return (t / scales.unsqueeze(2)).view(rows, -1).to(torch.float8_e4m3fn), scales


def _plain_weights(s, case):
    groups, inner, outer = case["groups"], case["inner"], case["outer"]
    nb, kb = _blocks(outer), _blocks(inner)
    w = torch.zeros((groups, BLOCK * nb, BLOCK * kb), device="cuda")
    w[:, :outer, :inner] = s["W"].float()
    t = w.view(groups, nb, BLOCK, kb, BLOCK)
    scales = _power_scales(t.abs().amax(dim=(2, 4)))
    codes = (t / scales.view(groups, nb, 1, kb, 1)).view_as(w).to(torch.float8_e4m3fn).view(torch.uint8)
    out = [codes[:, :outer].contiguous().view(torch.float8_e4m3fn), scales]
    if case["both"]:
        out += [codes.transpose(1, 2)[:, :inner].contiguous().view(torch.float8_e4m3fn), scales.transpose(1, 2).contiguous()]
    return out


def _values(codes, scales, inner):
    """Values of rows of codes, a scale to each block of each row."""
    rows = codes.shape[0]
    return (codes.float().view(rows, -1, BLOCK) * scales.unsqueeze(2)).view(rows, -1)[:, :inner]


def _plain_mm(s, case):
    dtype = TYPES[case["dtype"]]
    x = _values(*_plain_rows(s["X"]), case["inner"])
    Y = torch.empty((s["rows"], case["outer"]), dtype=dtype, device="cuda")
    out = [Y]
    if case["grad"]:
        d = _values(*_plain_rows(s["dY"]), case["outer"])
        out.append(torch.empty((s["rows"], case["inner"]), dtype=dtype, device="cuda"))
    for g in range(case["groups"]):
        a, b = s["bounds"][g], s["bounds"][g + 1]
        if a == b:
            continue
        w = _values(s["w_codes"][g], s["w_scales"][g].repeat_interleave(BLOCK, dim=0)[:case["outer"]], case["inner"])
        rows = x[a:b] if s["src"] is None else x[torch.div(s["src"][a:b], case["k"], rounding_mode="floor").long()]
        Y[a:b] = rows @ w.t()
        if case["grad"]:
            out[1][a:b] = d[a:b] @ w
    return out


def run(s):
    case = s["case"]
    op = case["op"]
    if not own:
        if op == "rows":
            return list(_plain_rows(s["X"]))
        return {"embed": _plain_embed, "balance": _plain_balance, "weights": _plain_weights, "mm": _plain_mm}[op](s, case)
    lib = s["lib"]
    if op == "embed":
        tokens, vocabulary, width = case["tokens"], case["vocabulary"], case["width"]
        for ids, out in zip(s["ids"], s["out"]):
            lib.sgap_embed(tokens, vocabulary, width, ids, s["W"], out, scale=case["scale"])
        if not case["steps"]:
            return list(s["out"])
        for i, (ids, dout) in enumerate(zip(s["ids"], s["dout"])):
            lib.sgap_embed_grad(tokens, vocabulary, width, ids, dout, s["dW"], scale=case["scale"], accumulate=i > 0, workspace=s["workspace"])
        return s["out"] + [s["dW"]]
    if op == "balance":
        sizes = case["tokens"], case["experts"], case["k"], case["sequences"]
        lib.sgap_route_balance(*sizes, s["logits"], s["experts"], s["segments"], s["loss"], s["counts"], s["rows"], workspace=s["workspace"])
        lib.sgap_route_balance_grad(*sizes, s["logits"], s["experts"], s["segments"], s["counts"], s["rows"], s["dloss"], s["dlogits"])
        return [s["loss"], s["counts"], s["rows"], s["dlogits"]]
    if op == "weights":
        lib.sgap_f8_weights(case["groups"], case["inner"], case["outer"], s["W"], s["codes"], s["scales"], s["codes_t"], s["scales_t"])
        return [s["codes"], s["scales"]] + ([s["codes_t"], s["scales_t"]] if case["both"] else [])
    if op == "rows":
        lib.sgap_f8_rows(case["rows"], case["inner"], s["X"], s["codes"], s["scales"])
        return [s["codes"], s["scales"]]
    groups, inner, outer, rows = case["groups"], case["inner"], case["outer"], s["rows"]
    gather = {} if s["src"] is None else {"src": s["src"], "src_div": case["k"]}
    lib.sgap_f8_rows(case["tokens"], inner, s["X"], s["x_codes"], s["x_scales"])
    lib.sgap_grouped_mm_f8(groups, rows, inner, outer, s["offsets"], s["x_codes"], s["x_scales"], s["w_codes"], s["w_scales"], s["Y"], **gather)
    if not case["grad"]:
        return [s["Y"]]
    lib.sgap_f8_rows(rows, outer, s["dY"], s["d_codes"], s["d_scales"])
    lib.sgap_grouped_mm_f8(groups, rows, outer, inner, s["offsets"], s["d_codes"], s["d_scales"], s["t_codes"], s["t_scales"], s["dX"])
    return [s["Y"], s["dX"]]


# --------------------------------------------------------------------------
# the definition in 64 bits
# --------------------------------------------------------------------------

def _exact_embed(s, case):
    W, scale = s["W"].double(), float(np.float32(case["scale"]))
    out, dW = [], None
    for ids, dout in zip(s["ids"], s["dout"]):
        real = torch.nonzero(ids >= 0)[:, 0]
        rows = torch.zeros(dout.shape, dtype=torch.float64, device="cuda")
        rows[real] = W[ids[real].long()] * scale
        out.append(rows)
        if case["steps"]:
            # tokens in the order of their ids; the sums between the places where a run of equal ids begins and ends
            sorted_ids, order = torch.sort(ids[real].long(), stable=True)
            seen, lengths = torch.unique_consecutive(sorted_ids, return_counts=True)
            upto = torch.cumsum(dout[real][order].double(), dim=0)
            ends = torch.cumsum(lengths, 0) - 1
            total = upto[ends]
            total[1:] -= upto[ends[:-1]]
            dW = torch.zeros(W.shape, dtype=torch.float64, device="cuda") if dW is None else dW
            dW[seen] += total * scale
    return out + ([] if dW is None else [dW])


def _exact_balance(s, case):
    experts, k, sequences = case["experts"], case["k"], case["sequences"]
    x, chosen = s["logits"].double().cpu().numpy(), s["experts"].cpu().numpy()
    counts, rows = np.zeros((sequences, experts), dtype=np.int32), np.zeros(sequences, dtype=np.int32)
    shares, p = np.zeros((sequences, experts)), np.zeros_like(x)
    some = chosen[:, 0] >= 0
    for i in range(sequences):
        at = np.arange(s["bounds"][i], s["bounds"][i + 1])
        at = at[some[at]]
        rows[i] = len(at)
        if len(at) == 0:
            continue
        p[at] = np.exp(x[at] - np.logaddexp.reduce(x[at], axis=1, keepdims=True))
        shares[i] = p[at].mean(axis=0)
        picked = chosen[at].reshape(-1)
        counts[i] = np.bincount(picked[picked >= 0], minlength=experts)
    used = max(int((rows > 0).sum()), 1)
    f = (counts.astype(np.int64) * experts - k * rows[:, None].astype(np.int64)) / (k * np.maximum(rows, 1)[:, None].astype(np.float64))
    loss = float(((f + 1) * shares).sum() / used)
    dlogits = np.zeros_like(x)
    for i in range(sequences):
        a, b = s["bounds"][i], s["bounds"][i + 1]
        if rows[i]:
            dlogits[a:b] = p[a:b] * f[i] - p[a:b] * (p[a:b] @ f[i])[:, None]
            dlogits[a:b] *= float(np.float32(0.01)) / (used * int(rows[i]))
    return [torch.tensor([loss], dtype=torch.float64), torch.from_numpy(counts), torch.from_numpy(rows), torch.from_numpy(dlogits)]


def _exact_codes(blocks, most):
    """(codes as numbers, scales) in 64 bits: steps of an e4m3 number at its own exponent, -6 at least, halves to even.  Powers of
    two out of tables: a device's pow() need not be exact."""
    powers = torch.tensor([2.0 ** e for e in range(-126, 122)], dtype=torch.float64, device="cuda")
    scales = powers[torch.searchsorted(powers * LARGEST, most.clamp(min=LARGEST * 2.0 ** -126).contiguous())]
    scales = torch.where(most > 0, scales, torch.ones_like(most))
    v = blocks / scales
    # |v| = m 2^e with m in [1/2, 1): eight steps from a half to one
    steps = torch.tensor([2.0 ** (e - 4) for e in range(-5, 10)], dtype=torch.float64, device="cuda")
    step = steps[torch.frexp(v)[1].long().clamp(-5, 9) + 5]
    step = torch.where(v == 0, steps[0], step)
    return torch.round(v / step) * step, scales


def _exact_rows(x):
    rows, inner = x.shape
    blocks = torch.nn.functional.pad(x.double(), (0, -inner % BLOCK)).view(rows, -1, BLOCK)
    codes, scales = _exact_codes(blocks, blocks.abs().amax(dim=2, keepdim=True))
    return codes.reshape(rows, -1), scales[:, :, 0]


def _exact_weights(s, case):
    groups, inner, outer = case["groups"], case["inner"], case["outer"]
    every, scales = [], []
    for g in range(groups):
        w = torch.nn.functional.pad(s["W"][g].double(), (0, -inner % BLOCK, 0, -outer % BLOCK))
        t = w.view(_blocks(outer), BLOCK, _blocks(inner), BLOCK)
        codes, scale = _exact_codes(t, t.abs().amax(dim=(1, 3), keepdim=True))
        every.append(codes.view_as(w).float())   # (numbers of eight bits: nothing is lost)
        scales.append(scale.view(_blocks(outer), _blocks(inner)))
    codes, scales = torch.stack(every), torch.stack(scales)
    out = [codes[:, :outer], scales]
    if case["both"]:
        out += [codes.permute(0, 2, 1)[:, :inner], scales.permute(0, 2, 1)]
    return [t.contiguous() for t in out]


def _exact_mm(s, case):
    inner, outer = case["inner"], case["outer"]

    def rows_of(x):
        codes, scales = _exact_rows(x)
        return (codes * scales.repeat_interleave(BLOCK, dim=1))[:, :x.shape[1]].contiguous()

    token = torch.arange(s["rows"], device="cuda") if s["src"] is None else torch.div(s["src"].long(), case["k"], rounding_mode="floor")
    X = rows_of(s["X"])
    out = [torch.zeros((s["rows"], outer), dtype=torch.float64, device="cuda")]
    if case["grad"]:
        D = rows_of(s["dY"])
        out.append(torch.zeros((s["rows"], inner), dtype=torch.float64, device="cuda"))
    for g, (a, b) in enumerate(zip(s["bounds"], s["bounds"][1:])):
        if b == a:
            continue
        scales = s["w_scales"][g].double().repeat_interleave(BLOCK, dim=0)[:outer].repeat_interleave(BLOCK, dim=1)[:, :inner]
        w = (s["w_codes"][g].double()[:, :inner] * scales).contiguous()
        out[0][a:b] = torch.mm(X[token[a:b]], w.t().contiguous())
        if case["grad"]:
            out[1][a:b] = torch.mm(D[a:b].contiguous(), w)
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "rows":
        return list(_exact_rows(s["X"]))
    return {"embed": _exact_embed, "balance": _exact_balance, "weights": _exact_weights, "mm": _exact_mm}[case["op"]](s, case)


# --------------------------------------------------------------------------
# what a pass cannot do without
# --------------------------------------------------------------------------

def _missed(kinds, share_of):
    """Kinds that nothing of a batch is, in the mean, of `kinds`, where share_of(i) is the chance that it has kind i."""
    return float(np.sum(share_of(np.arange(kinds))))


def work(case):
    size = BYTES[case["dtype"]]
    if case["op"] == "embed":
        tokens, vocabulary, width, steps = case["tokens"], case["vocabulary"], case["width"], case["steps"]
        # rows of the table that some token has (frequencies as prepare() draws them)
        chance = lambda i: (1 - np.log((i + 2) / (i + 1)) / math.log(vocabulary + 1)) ** tokens  # noqa: E731
        seen = vocabulary - _missed(vocabulary, chance)
        moved = max(steps, 1) * (tokens * 4 + seen * width * size + tokens * width * size)
        if steps:
            moved += steps * (tokens * 4 + tokens * width * size) + vocabulary * width * BYTES[case["grad_dtype"]]
        return {"bytes": moved, "flops": tokens * width * max(steps, 1) * (2 if steps else 1)}
    if case["op"] == "balance":
        tokens, experts, k, sequences = case["tokens"], case["experts"], case["k"], case["sequences"]
        return {"bytes": 2 * tokens * experts * size + tokens * k * 4 + sequences * (experts + 2) * 4 + 8, "flops": 12 * tokens * experts}
    if case["op"] == "weights":
        elements = case["groups"] * case["inner"] * case["outer"]
        blocks = case["groups"] * _blocks(case["inner"]) * _blocks(case["outer"])
        return {"bytes": elements * size + (elements + blocks * 4) * (2 if case["both"] else 1), "flops": 2 * elements}
    if case["op"] == "rows":
        elements = case["rows"] * case["inner"]
        return {"bytes": elements * (size + 1) + case["rows"] * _blocks(case["inner"]) * 4, "flops": 2 * elements}
    groups, tokens, k, inner, outer = case["groups"], case["tokens"], case["k"], case["inner"], case["outer"]
    rows = tokens * max(k, 1)
    # groups that have a row, alike groups taken for unlike ones
    used = groups * (1 - ((1 - k / groups) ** tokens if k else (1 - 1 / groups) ** tokens))
    weights = used * (inner * outer + _blocks(inner) * _blocks(outer) * 4)
    moved = (groups + 1) * 4 + (rows * 4 if k else 0) + tokens * inner * size + weights + rows * outer * size
    if case["grad"]:
        moved += rows * outer * size + weights + rows * inner * size
    return {"bytes": moved, "flops": 2 * rows * inner * outer * (2 if case["grad"] else 1)}
