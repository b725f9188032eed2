"""Plain 64-bit forms of the operators of a mixture of experts, and the bounds their results are held to.

u: half a unit in the last place of the result's type, for the one rounding when it is stored.  e: what a sum in 32 bits may
lose per addition, 2^-23 (twice the rounding to nearest, so that an instruction that cuts off passes).  A sum of n products is
then within (n + 4) * e of the sum of the products' magnitudes."""
import numpy as np
import torch

U = {torch.float32: 2.0**-24, torch.float16: 2.0**-11, torch.bfloat16: 2.0**-8}
TINY = {torch.float32: 2.0**-149, torch.float16: 2.0**-24, torch.bfloat16: 2.0**-133}
E = 2.0**-23


def assert_within(got, want, slack, what=""):
    """|got - want| <= slack + rounding of the result, element by element; infinities and NaN have to be the same ones."""
    dtype = got.dtype
    g, w = got.detach().double().cpu().numpy(), want.numpy() if torch.is_tensor(want) else want
    s = slack.numpy() if torch.is_tensor(slack) else slack
    assert g.shape == w.shape, what
    odd = ~np.isfinite(w)
    np.testing.assert_array_equal(g[odd], w[odd], err_msg=what)
    bound = s + U[dtype] * (np.abs(w) + s) + TINY[dtype]
    off = (~odd) & ~(np.abs(g - w) <= bound)
    if off.any():
        at = tuple(np.argwhere(off)[0])
        raise AssertionError(f"{what}: {int(off.sum())} of {off.size} elements off, first at {at}: got {g[at]!r}, want {w[at]!r}, "
                             f"bound {np.broadcast_to(bound, w.shape)[at]!r}")


def random(seed, *shape, dtype=torch.float32, scale=1.0):
    gen = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=gen) * scale).to(dtype)


def offsets_of(sizes):
    return torch.from_numpy(np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32))


def source_rows(R, x_rows, src, src_div):
    """Row of X of each row (x_rows: none)."""
    if src is None:
        return torch.arange(R)
    rows = torch.div(src.long(), src_div, rounding_mode="floor")
    return torch.where((rows < 0) | (rows >= x_rows), torch.full_like(rows, x_rows), rows)


def grouped_mm(offsets, X, W, layout, R, src=None, src_div=1):
    """(Y, sum of magnitudes): W is G x N x K or G x K x N."""
    x = torch.cat([X.double(), torch.zeros(1, X.shape[1], dtype=torch.float64)])[source_rows(R, X.shape[0], src, src_div)]
    w = W.double() if layout == "nk" else W.double().transpose(1, 2)
    Y, B = (torch.zeros(R, w.shape[1], dtype=torch.float64) for _ in range(2))
    for g in range(w.shape[0]):
        a, b = int(offsets[g]), int(offsets[g + 1])
        Y[a:b] = x[a:b] @ w[g].t()
        B[a:b] = x[a:b].abs() @ w[g].abs().t()
    return Y, B


def grouped_wgrad(offsets, X, dY, layout, src=None, src_div=1):
    R = dY.shape[0]
    x = torch.cat([X.double(), torch.zeros(1, X.shape[1], dtype=torch.float64)])[source_rows(R, X.shape[0], src, src_div)]
    d = dY.double()
    out, bound = [], []
    for g in range(len(offsets) - 1):
        a, b = int(offsets[g]), int(offsets[g + 1])
        l, r = (d, x) if layout == "nk" else (x, d)
        out.append(l[a:b].t() @ r[a:b])
        bound.append(l[a:b].abs().t() @ r[a:b].abs())
    return torch.stack(out), torch.stack(bound)


def route(logits, k, renormalise):
    """gates, experts, slot, order, offsets of sgap_route_topk, row by row."""
    x = logits.double().numpy()
    T, n = x.shape
    gates, experts = np.zeros((T, k)), np.full((T, k), -1, dtype=np.int32)
    for t in range(T):
        key = np.where(np.isnan(x[t]), np.inf, x[t])  # NaN before +inf: by the second key
        ranked = sorted((e for e in range(n) if not x[t, e] == -np.inf), key=lambda e: (not np.isnan(x[t, e]), -key[e], e))[:k]
        if not ranked:
            continue
        with np.errstate(invalid="ignore"):
            p = np.exp(x[t] - x[t, ranked[0]])
            total = p[ranked].sum() if renormalise else p.sum()
            gates[t, :len(ranked)] = p[ranked] / total
        experts[t, :len(ranked)] = ranked
    pairs = sorted((int(e), p) for p, e in enumerate(experts.reshape(-1)) if e >= 0)
    order, slot = np.full(T * k, -1, dtype=np.int32), np.full(T * k, -1, dtype=np.int32)
    for at, (_, p) in enumerate(pairs):
        order[at], slot[p] = p, at
    counts = np.bincount([e for e, _ in pairs], minlength=n) if pairs else np.zeros(n, dtype=np.int64)
    return gates, experts, slot.reshape(T, k), order, np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)


def route_grad(logits, gates, experts, dgates, renormalise):
    """(dlogits, sum of magnitudes) by the gates' Jacobian."""
    x = logits.double().numpy()
    T, n = x.shape
    out, size = np.zeros((T, n)), np.zeros((T, n))
    for t in range(T):
        there = experts[t] >= 0
        if not there.any():
            continue
        e, g, d = experts[t][there], gates[t][there], dgates[t][there]
        p = np.zeros(n)
        if renormalise:
            p[e] = g
        else:
            finite = x[t] > -np.inf
            p[finite] = np.exp(x[t][finite] - x[t].max())
            p /= p.sum()
        for j in range(len(e)):
            out[t] -= g[j] * d[j] * p
            size[t] += abs(g[j] * d[j]) * p
            out[t, e[j]] += g[j] * d[j]
            size[t, e[j]] += abs(g[j] * d[j])
    return out, size


def w4_weights(codes, scales, zeros, group_k):
    """G x N x K in 64 bits."""
    c = codes.long()
    w = torch.stack([c % 16, c // 16], dim=3).flatten(2).double()
    zero = torch.full_like(scales, 8).double() if zeros is None else zeros.double()
    return (w - zero.repeat_interleave(group_k, dim=2)) * scales.double().repeat_interleave(group_k, dim=2)


def w4_bound(codes, scales, zeros, group_k):
    """Weights of the magnitudes that the kernel sums: a code counts as 16 more, and so does its zero point."""
    c = codes.long()
    w = torch.stack([c % 16, c // 16], dim=3).flatten(2).double()
    zero = torch.full_like(scales, 8).double() if zeros is None else zeros.double()
    return (32 + w + zero.repeat_interleave(group_k, dim=2)) * scales.double().abs().repeat_interleave(group_k, dim=2)
