"""The calls that a model of tokens makes beside those of experts_on_host, on host tensors in torch's own operations."""
import torch

import experts_on_host
import tokens_util
from paper_2209_02882_amd import binding


class Calls(experts_on_host.Calls):
    SGAP_F8_BLOCK = tokens_util.BLOCK

    def __getattr__(self, name):
        if name in ("sgap_route_balance_workspace_size", "sgap_embed_grad_workspace_size"):
            return lambda *args: 0
        step = HERE.get(name)
        if step is None:
            return super().__getattr__(name)

        def call(*args, **kwargs):
            self.append(name)
            with torch.no_grad():
                step(*args, **kwargs)

        return call


def on_host(monkeypatch):
    """The calls of the binding that a model makes from here on."""
    from paper_2209_02882_amd import experts

    calls = Calls()
    monkeypatch.setattr(experts, "binding", calls)
    return calls


def route_balance(T, E, k, S, logits, experts, segments, loss, counts, rows, workspace=None):
    value, c, n, _, _ = tokens_util.balance(logits, experts, segments, k)
    loss.fill_(float(value))
    counts.copy_(torch.from_numpy(c))
    rows.copy_(torch.from_numpy(n))


def route_balance_grad(T, E, k, S, logits, experts, segments, counts, rows, dloss, dlogits, accumulate=False):
    grad = torch.from_numpy(tokens_util.balance(logits, experts, segments, k)[3]) * dloss.double()
    dlogits.copy_(dlogits.double() + grad if accumulate else grad)


def embed(T, V, D, ids, weights, out, scale=1.0):
    out.copy_(tokens_util.embed(ids, weights, scale))


def embed_grad(T, V, D, ids, dout, dweights, scale=1.0, accumulate=False, workspace=None):
    grad = tokens_util.embed_grad(ids, dout, V, scale)[0]
    dweights.copy_(dweights.double() + grad if accumulate else grad)


def keep(codes, scales, numbers):
    codes.copy_(torch.from_numpy(numbers[0]).float().to(torch.float8_e4m3fn))
    scales.copy_(torch.from_numpy(numbers[1]))


def f8_rows(R, K, X, codes, scales):
    keep(codes, scales, tokens_util.f8_rows(X))


def f8_weights(G, K, N, W, codes, scales, codes_t=None, scales_t=None):
    keep(codes, scales, tokens_util.f8_weights(W))
    if codes_t is not None:
        keep(codes_t, scales_t, tokens_util.f8_weights(W.transpose(1, 2)))


def grouped_mm_f8(G, R, K, N, offsets, X, x_scales, W, w_scales, Y, src=None, src_div=1):
    x = experts_on_host.rows_of(tokens_util.values(X, x_scales, K, True), R, src, src_div)
    w = tokens_util.values(W, w_scales, K, False)
    for g in range(G):
        a, b = int(offsets[g]), int(offsets[g + 1])
        Y[a:b] = (x[a:b] @ w[g].t()).to(Y.dtype)


HERE = {"sgap_" + step.__name__: step for step in (route_balance, route_balance_grad, embed, embed_grad, f8_rows, f8_weights,
                                                   grouped_mm_f8)}
assert all(hasattr(binding, name) for name in HERE) and binding.SGAP_F8_BLOCK == Calls.SGAP_F8_BLOCK
