"""Plain 64-bit forms of embeddings, the balance loss and numbers of 8 bits, on the host (see experts_util for the bounds' words)."""
import numpy as np
import torch

BLOCK = 128


def blocks(n):
    return (n + BLOCK - 1) // BLOCK


def embed(ids, weights, scale):
    """out: T x D in 64 bits."""
    w, V = weights.double(), weights.shape[0]
    out = torch.zeros(len(ids), w.shape[1], dtype=torch.float64)
    real = [t for t, i in enumerate(ids.tolist()) if 0 <= i < V]
    out[real] = w[ids[real].long()] * scale
    return out


def embed_grad(ids, dout, V, scale):
    """(gradient, sum of magnitudes, tokens) of the table's rows."""
    d = dout.double()
    grad, size = torch.zeros(V, d.shape[1], dtype=torch.float64), torch.zeros(V, d.shape[1], dtype=torch.float64)
    tokens = torch.zeros(V, 1, dtype=torch.float64)
    real = torch.tensor([0 <= i < V for i in ids.tolist()], dtype=torch.bool)
    at = ids[real].long()
    grad.index_add_(0, at, d[real] * scale)
    size.index_add_(0, at, (d[real] * scale).abs())
    tokens.index_add_(0, at, torch.ones(int(real.sum()), 1, dtype=torch.float64))
    return grad, size, tokens


def balance(logits, experts, segments, k):
    """(loss, counts, rows, gradient of the logits, its magnitudes), sequence by sequence."""
    x, chosen = logits.double().numpy(), experts.numpy()
    T, E = x.shape
    bounds = [0, T] if segments is None else segments.tolist()
    S = len(bounds) - 1
    counts, rows = np.zeros((S, E), dtype=np.int32), np.zeros(S, dtype=np.int32)
    p, f1, losses = np.zeros((T, E)), np.zeros((S, E)), np.zeros(S)
    for s in range(S):
        mine = [t for t in range(bounds[s], bounds[s + 1]) if any(0 <= e < E for e in chosen[t])]
        rows[s] = len(mine)
        for t in mine:
            for e in chosen[t]:
                if 0 <= e < E:
                    counts[s, e] += 1
            with np.errstate(invalid="ignore"):
                q = np.exp(x[t] - x[t].max())
            p[t] = q / q.sum()
        if mine:
            f1[s] = (counts[s].astype(np.int64) * E - k * len(mine)) / (k * len(mine))
            losses[s] = ((1 + f1[s]) * p[mine].mean(axis=0)).sum()
    used = int((rows > 0).sum())
    grad, size = np.zeros((T, E)), np.zeros((T, E))
    for s in range(S):
        a, b = bounds[s], bounds[s + 1]
        if rows[s]:
            scale = 1.0 / (used * int(rows[s]))
            grad[a:b] = scale * p[a:b] * (f1[s] - (p[a:b] @ f1[s])[:, None])
            size[a:b] = scale * p[a:b] * (np.abs(f1[s]) + (p[a:b] @ np.abs(f1[s]))[:, None])
    return losses.sum() / max(used, 1), counts, rows, grad, size


def e4m3(v):
    """The nearest e4m3 number (ties to even) of 64-bit values of magnitude 448 or less; NaN stays."""
    _, e = np.frexp(v)
    step = np.ldexp(1.0, np.maximum(e - 1, -6) - 3)
    return np.round(v / step) * step


def power_scale(most):
    """The smallest power of two, 2^-126 at least, that brings `most` to 448 or less; 1 for 0."""
    s = np.ones_like(most)
    m, e = np.frexp(most / 448.0)
    s[most > 0] = np.ldexp(1.0, np.maximum(np.where(m == 0.5, e - 1, e), -126))[most > 0]
    return s


def f8(tiles, axes):
    """(codes, scales) of tiles whose `axes` share a scale."""
    finite = np.isfinite(tiles)
    scales = power_scale(np.where(finite, np.abs(tiles), 0).max(axis=axes, keepdims=True))
    return e4m3(np.where(finite, tiles, np.nan) / scales), scales


def f8_rows(x):
    """(codes R x whole blocks, scales R x blocks) in 64 bits."""
    x = x.double().numpy()
    R, K = x.shape
    whole = np.zeros((R, blocks(K) * BLOCK))
    whole[:, :K] = x
    codes, scales = f8(whole.reshape(R, -1, BLOCK), (2,))
    return codes.reshape(R, -1), scales.reshape(R, -1)


def f8_weights(w):
    """(codes G x N x whole blocks of K, scales) in 64 bits."""
    w = w.double().numpy()
    G, N, K = w.shape
    whole = np.zeros((G, blocks(N) * BLOCK, blocks(K) * BLOCK))
    whole[:, :N, :K] = w
    codes, scales = f8(whole.reshape(G, blocks(N), BLOCK, blocks(K), BLOCK), (2, 4))
    return codes.reshape(whole.shape)[:, :N], scales.reshape(G, blocks(N), blocks(K))


def values(codes, scales, K, per_row):
    """Values in 64 bits of codes (.. x N x whole blocks) with scales for each row, or for 128 rows."""
    c, s = codes.double(), scales.double()
    if not per_row:
        s = s.repeat_interleave(BLOCK, dim=-2)[..., :c.shape[-2], :]
    return (c * s.repeat_interleave(BLOCK, dim=-1))[..., :K]


def random_codes(gen, *shape, K):
    """Any finite e4m3 numbers in rows of whole blocks, zeros from column K on."""
    bits = torch.randint(0, 256, shape, generator=gen, dtype=torch.int64)
    bits = torch.where((bits & 127) == 127, bits - 1, bits).to(torch.uint8)
    bits[..., K:] = 0
    return bits.view(torch.float8_e4m3fn)


def filled(dtype, *shape):
    """Device memory that holds what no result is: NaN, or a negative count."""
    if dtype == torch.float8_e4m3fn:
        return torch.full(shape, 0xff, dtype=torch.uint8, device="cuda").view(dtype)
    return torch.full(shape, -77 if dtype == torch.int32 else float("nan"), dtype=dtype, device="cuda")
