"""The model of tokens and the layer in 8 bits: what they differentiate, ask for and keep.  The library's calls are torch's here.
No GPU."""
import pytest
import torch

import tokens_util as tu
from paper_2209_02882_amd import experts
from tokens_on_host import on_host

V, WIDTH, HIDDEN, E, K = 11, 136, 24, 4, 2
SEGMENTS = [[0, 0, 9, 20], None]


def model_and_ids(eight_bits, tokens=23):
    torch.manual_seed(4)
    model = experts.TokenModel(V, WIDTH, HIDDEN, E, K, dtype=torch.float32, device="cpu", eight_bits=eight_bits)
    return model, torch.randint(-2, V + 2, (tokens,), dtype=torch.int32)


class Product8(torch.autograd.Function):
    """x @ w^T of 8-bit numbers of both, dx out of those of the gradient and the weights the other way round, dw in full."""

    @staticmethod
    def forward(ctx, x, w):
        ctx.save_for_backward(x, w)
        return rounded(x) @ rounded(w, weights=True).t()

    @staticmethod
    def backward(ctx, dy):
        x, w = ctx.saved_tensors
        return rounded(dy) @ rounded(w.t().contiguous(), weights=True).t(), dy.t() @ x


def rounded(x, weights=False):
    if not x.numel():
        return x
    codes, scales = tu.f8_weights(x[None]) if weights else tu.f8_rows(x)
    return tu.values(torch.from_numpy(codes), torch.from_numpy(scales), x.shape[1], not weights).view(x.shape)


def plain(model, ids, segments, eight_bits):
    """(logits, balance) in 64 bits by torch's autograd, one expert after the other."""
    product = Product8.apply if eight_bits else lambda x, w: x @ w.t()
    layer, table, there = model.layer, model.embedding.weights, (ids >= 0) & (ids < V)
    x = torch.where(there[:, None], table[ids.clamp(0, V - 1).long()], 0) * model.embedding.scale
    scores = x @ layer.router.t()
    top, chosen = (v[:, :K] for v in torch.sort(scores, dim=1, descending=True, stable=True))  # the first of equal ones
    gates, out = torch.softmax(top, dim=1), torch.zeros_like(x)
    for e in range(E):
        t, j = (chosen == e).nonzero(as_tuple=True)
        h = experts.gated(product(x[t], layer.up[e]))
        out = out.index_add(0, t, product(h, layer.down[e]) * gates[t, j, None])
    bounds = segments.tolist() if segments is not None else [0, len(ids)]
    losses = []
    for a, b in zip(bounds, bounds[1:]):
        if b > a:
            f = torch.bincount(chosen[a:b].reshape(-1), minlength=E).double() * E / (K * (b - a))
            losses.append((f * torch.softmax(scores[a:b], dim=1).mean(0)).sum())
    return (x + out) @ table.t(), sum(losses) / len(losses)


# the same numbers of 32 bits in both, tokens whose experts are equal among them (tokens outside the table: zeros), and sums of
# at most 136 products in 32 bits: 2^-24 * 136 * the 5 sums one after the other, 2^-14 of the largest value.  In 8 bits that
# takes a number to the other side of a code's edge now and then, one 2^-3 of itself away, of 136 and more that are summed: at
# most one in a hundred may do so, for 2^-3 * (1 / 100)^(1/2) = 2^-6 of the norm
@pytest.mark.parametrize("eight_bits", [False, True])
@pytest.mark.parametrize("bounds", SEGMENTS)
def test_the_calls_on_the_host_are_the_model(bounds, eight_bits, monkeypatch):
    on_host(monkeypatch)
    model, ids = model_and_ids(eight_bits)
    segments = None if bounds is None else torch.tensor(bounds, dtype=torch.int32)
    twin = experts.TokenModel(V, WIDTH, HIDDEN, E, K, dtype=torch.float64, device="cpu")
    twin.load_state_dict(model.state_dict())
    weight = torch.randn(len(ids), V)
    results = []
    for logits, balance, params in ((*model(ids, segments), model.parameters()),
                                    (*plain(twin, ids, segments, eight_bits), twin.parameters())):
        loss = (logits * weight).sum() + 3 * balance
        results.append([logits, balance, *torch.autograd.grad(loss, list(params))])
    for got, want in zip(*results):
        off = got.double() - want
        assert off.norm() <= 2.0**-6 * want.norm() if eight_bits else off.abs().max() <= 2.0**-14 * want.abs().max()


@pytest.mark.parametrize("wrt", ["table", "router", "up", "down"])
def test_second_derivatives_are_refused(wrt, monkeypatch):
    on_host(monkeypatch)
    model, ids = model_and_ids(True)
    logits, balance = model(ids)
    loss = logits.square().sum() + balance
    of = {"table": model.embedding.weights, "router": model.layer.router, "up": model.layer.up, "down": model.layer.down}[wrt]
    (grad,) = torch.autograd.grad(loss, of, create_graph=True)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        (loss + grad.square().sum()).backward()


@pytest.mark.parametrize("frozen", ["", "experts", "table", "table and up"])
def test_gradients_that_nobody_asks_for_are_not_computed(frozen, monkeypatch):
    calls = on_host(monkeypatch)
    model, ids = model_and_ids(True)
    for name, part in (("table", model.embedding.weights), ("up", model.layer.up), ("down", model.layer.down)):
        part.requires_grad_(name not in frozen and not (frozen == "experts" and name != "table"))
    logits, balance = model(ids)
    made = {name: calls.count(name) for name in set(calls)}
    assert made == {"sgap_embed": 1, "sgap_route_topk": 1, "sgap_route_balance": 1, "sgap_f8_rows": 2, "sgap_f8_weights": 2,
                    "sgap_grouped_mm_f8": 2, "sgap_route_combine": 1}
    del calls[:]
    (logits.square().sum() + balance).backward()
    made = {name: calls.count(name) for name in set(calls)}
    want = {"sgap_route_combine_grad": 1, "sgap_route_topk_grad": 1, "sgap_route_balance_grad": 1}
    through_both = {"sgap_f8_rows": 2, "sgap_grouped_mm_f8": 2, "sgap_route_combine": 1, "sgap_embed_grad": 1}
    if frozen in ("", "experts"):
        want |= through_both | ({} if frozen else {"sgap_grouped_mm_wgrad": 2})
    elif frozen == "table":
        want |= {"sgap_f8_rows": 1, "sgap_grouped_mm_f8": 1, "sgap_grouped_mm_wgrad": 2}
    else:
        want |= {"sgap_grouped_mm_wgrad": 1}
    assert made == want


def test_transposed_codes_are_made_only_for_a_gradient_of_the_rows(monkeypatch):
    on_host(monkeypatch)
    made = []
    weights8 = experts.Weights8
    monkeypatch.setattr(experts, "Weights8", lambda weights, both=False: made.append(both) or weights8(weights, both))
    model, ids = model_and_ids(True)
    model.embedding.weights.requires_grad_(False)
    model(ids)
    assert made == [False, True]  # the rows between the products have one


# a loss that is not used has no gradient: the other one is what it would be alone
def test_without_the_balance_loss_the_gradient_is_the_routers(monkeypatch):
    on_host(monkeypatch)
    model, ids = model_and_ids(False)
    x = model.embedding(ids).detach()
    grads = []
    for out in (model.layer(x), model.layer.balanced(x)[0]):
        grads.append(torch.autograd.grad(out.square().sum(), list(model.layer.parameters())))
    for a, b in zip(*grads):
        assert torch.equal(a, b)


def test_ids_of_any_shape(monkeypatch):
    on_host(monkeypatch)
    model, ids = model_and_ids(False, 24)
    flat = model.embedding(ids)
    assert torch.equal(model.embedding(ids.view(2, 3, 4)), flat.view(2, 3, 4, WIDTH))
    assert torch.equal(model.embedding(ids.view(4, 6).t()), flat.view(4, 6, WIDTH).transpose(0, 1))
    assert model.embedding(ids[:0]).shape == (0, WIDTH)


@pytest.mark.parametrize("bits", [0, 3, 16])
def test_bits_that_no_call_serves(bits):
    layer = experts.ExpertLayer(16, 8, 4, 2, device="cpu")
    with pytest.raises(ValueError, match="4 or 8"):
        layer.quantise(bits=bits)
    assert layer.served is None


def test_serving_in_8_bits_is_the_layer_in_8_bits(monkeypatch):
    calls = on_host(monkeypatch)
    torch.manual_seed(5)
    layer = experts.ExpertLayer(140, 9, E, K, dtype=torch.float32, device="cpu", eight_bits=True)
    x = torch.randn(7, 140)
    want = layer(x).detach()
    layer.quantise(bits=8)
    del calls[:]
    assert torch.equal(layer.serve(x), want)
    assert "sgap_f8_weights" not in calls  # laid out once
