"""A run of embedding, routing with its balance loss, products in 8 bits and the sums by token, forth and back, as a model makes it."""
import pytest
import torch

import tokens_util as tu
from paper_2209_02882_amd import experts

pytestmark = pytest.mark.gpu


def ids_of(T, V, low=-2, high=2):
    return torch.randint(low, V + high, (T,), device="cuda", dtype=torch.int32)


def plain(model, ids, segments, k):
    """(logits, balance) in 64 bits, one expert after the other; the tokens of no sequence count for no balance."""
    layer, table = model.layer, model.embedding.weights
    V, E = table.shape[0], layer.up.shape[0]
    there = (ids >= 0) & (ids < V)
    x = torch.where(there[:, None], table[ids.clamp(0, V - 1).long()], 0) * model.embedding.scale
    scores = x @ layer.router.t()
    top, chosen = (v[:, :k] for v in torch.sort(scores, dim=1, descending=True, stable=True))
    gates, out = torch.softmax(top, dim=1), torch.zeros_like(x)
    for e in range(E):
        h = experts.gated(x @ layer.up[e].t()) @ layer.down[e].t()
        out = out + h * torch.where(chosen == e, gates, torch.zeros_like(gates)).sum(1, keepdim=True)
    bounds = segments.tolist() if segments is not None else [0, len(ids)]
    losses = []
    for a, b in zip(bounds, bounds[1:]):
        if b > a:
            f = torch.zeros(E, dtype=torch.float64, device="cuda").scatter_add_(
                0, chosen[a:b].reshape(-1), torch.ones((b - a) * k, dtype=torch.float64, device="cuda")) * E / (k * (b - a))
            losses.append((f * torch.softmax(scores[a:b], dim=1).mean(0)).sum())
    return (x + out) @ table.t(), sum(losses) / len(losses)


# with products in 32 bits: chains of at most 5 sums of under 512 products, 2^-24 * 512 * 5 of the largest value
@pytest.mark.parametrize("bounds", [[0, 50, 50, 51, 90], None])
@pytest.mark.parametrize("V,width,hidden,E,k", [(70, 64, 48, 6, 2), (500, 33, 17, 5, 1), (3, 40, 24, 4, 4)])
def test_gradients_of_the_model(V, width, hidden, E, k, bounds):
    torch.manual_seed(V)
    model = experts.TokenModel(V, width, hidden, E, k, dtype=torch.float32, eight_bits=False)
    twin = experts.TokenModel(V, width, hidden, E, k, dtype=torch.float64)
    twin.load_state_dict(model.state_dict())
    ids, weight = ids_of(100, V), torch.randn(100, V, device="cuda")
    segments = None if bounds is None else torch.tensor(bounds, device="cuda", dtype=torch.int32)
    results = []
    for of, (logits, balance) in ((model, model(ids, segments)), (twin, plain(twin, ids, segments, k))):
        loss = (logits * weight).sum() + 3 * balance
        results.append([logits, balance, *torch.autograd.grad(loss, list(of.parameters()))])
    for got, want in zip(*results):
        assert (got.double() - want).abs().max() <= 2560 * 2.0**-24 * want.abs().max()


# A product in 8 bits and the gradient of its rows against the product of the full numbers: each number of either operand is
# off by half a step of 3 bits, 2^-4 of it, or of the smallest step, 2^-10 of its block's scale, which is under 2 / 448 of the
# block's largest; the result once more by half a step of its own type, and by 7 * 2^-13 of the sum (the bits that the
# instruction leaves out).  Numbers under a type's smallest normal one are multiples of eps times that (2^-24 in fp16, where a
# product of two such small gradients comes to lie): a result among them is off by half of one, without regard to its size.
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("gathered", [True, False])
@pytest.mark.parametrize("T,width,columns,E,k", [(130, 128, 96, 4, 2), (7, 200, 56, 5, 2), (520, 136, 264, 3, 1)])
def test_the_product_in_8_bits_is_near_the_product(T, width, columns, E, k, gathered, dtype):
    torch.manual_seed(T)
    gates, slot, order, offsets = experts.Route.apply(torch.randn(T, E, device="cuda"), k)
    x = torch.randn(T if gathered else T * k, width, device="cuda").to(dtype).requires_grad_()
    w = torch.randn(E, columns, width, device="cuda").to(dtype).requires_grad_()
    dy = torch.randn(T * k, columns, device="cuda").to(dtype)
    y = experts.GroupedMM8.apply(x, w, offsets, order, slot, gathered)
    dx, dw = torch.autograd.grad(y, (x, w), dy)
    src = (order // k if gathered else torch.arange(T * k, device="cuda")).long()
    x64, w64, dy64, ends = x.detach().double()[src], w.detach().double(), dy.double(), offsets.tolist()
    half = torch.finfo(dtype).eps / 2
    last = half * torch.finfo(dtype).tiny

    def bound(a, b):
        floor = lambda v: 2.0**-4 * v.abs() + 2.0**-10 / 224 * v.abs().max()  # noqa: E731
        off = floor(a) @ (b.abs() + floor(b)).t() + a.abs() @ floor(b).t()
        size = (a.abs() + floor(a)) @ (b.abs() + floor(b)).t()
        return off + size * (half + 7 * 2.0**-13) + last

    rows, limit = torch.zeros(T * k, width, device="cuda").double(), torch.zeros(T * k, width, device="cuda").double()
    for e in range(E):
        a, b = ends[e], ends[e + 1]
        assert ((y[a:b].double() - x64[a:b] @ w64[e].t()).abs() <= bound(x64[a:b], w64[e])).all() if b > a else True
        if b > a:
            w_t = w64[e].t().contiguous()
            rows[a:b], limit[a:b] = dy64[a:b] @ w64[e], bound(dy64[a:b], w_t)
        exact, size = dy64[a:b].t() @ x64[a:b], dy64[a:b].abs().t() @ x64[a:b].abs()
        assert ((dw[e].double() - exact).abs() <= (half + (b - a) * 2.0**-23) * size + last).all()  # sums of products in 32 bits
    if gathered:
        want, most = torch.zeros(T, width, device="cuda").double(), torch.zeros(T, width, device="cuda").double()
        want.index_add_(0, src, rows)
        most.index_add_(0, src, limit * (1 + 2 * half) + rows.abs() * 2 * half + last)  # the sum of k rounded rows is rounded too
        rows, limit = want, most
    assert ((dx.double() - rows).abs() <= limit).all()


# rounded as the calls by themselves: a logit less the largest by its size times 2^-24, exp, and sums over experts and tokens
def test_the_balance_loss_alone_has_its_gradient():
    torch.manual_seed(2)
    T, E, k = 300, 8, 2
    logits = (torch.randn(T, E, device="cuda") + torch.linspace(0, 2, E, device="cuda")).requires_grad_()
    *_, loss, counts = experts.RouteBalanced.apply(logits, k, None)
    (grad,) = torch.autograd.grad(loss, logits)
    on_host = logits.detach().cpu()
    chosen = torch.sort(on_host, dim=1, descending=True, stable=True)[1][:, :k].int()
    want, c, _, wanted, size = tu.balance(on_host, chosen, None, k)
    wide = float(on_host.max() - on_host.min())
    assert torch.equal(counts.cpu(), torch.from_numpy(c))
    assert abs(loss.item() - want) <= (T + E + wide + 16) * 2.0**-23 * want
    assert (abs(grad.double().cpu().numpy() - wanted) <= (2 * E + 2 * wide + 24) * 2.0**-23 * size).all()


def step_of(model, ids, segments):
    dlogits = torch.randn(len(ids), model.embedding.weights.shape[0], device="cuda").bfloat16()
    dbalance = torch.full((), 0.1, device="cuda")

    def step():
        logits, balance = model(ids, segments)
        grads = torch.autograd.grad((logits, balance), list(model.parameters()), (dlogits, dbalance))
        return logits.detach(), balance.detach(), *grads
    return step


# Two steps captured on a stream of their own, replayed in turn with eager work between: the same bits as the eager steps
# for new tokens and new sequences, whatever the replays before left in the workspaces.
def test_captured_steps_are_the_eager_ones():
    torch.manual_seed(3)
    V, T = 300, 160
    model = experts.TokenModel(V, 136, 72, 6, 2)
    other = experts.TokenModel(V, 64, 64, 4, 1)
    ids = ids_of(T, V, 0, 0)
    segments = torch.tensor([0, 100, 100, 160], device="cuda", dtype=torch.int32)
    steps = [step_of(m, ids, segments) for m in (model, other)]
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        for step in steps:
            step()
    torch.cuda.current_stream().wait_stream(stream)
    graphs, outs = [], []
    for step in steps:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=stream):
            outs.append(step())
    for turn in range(4):
        ids.copy_(ids_of(T, V, -1 if turn else 0, 1 if turn else 0))
        segments.copy_(torch.tensor([0, 20 * turn, 100 + turn, 160 - turn], dtype=torch.int32))
        for graph in graphs if turn % 2 else graphs[::-1]:
            graph.replay()
        torch.cuda.synchronize()
        for step, out in zip(steps, outs):
            for got, want in zip(out, step()):
                assert torch.equal(got, want)


def test_steps_on_another_stream_are_the_same():
    torch.manual_seed(4)
    model = experts.TokenModel(200, 128, 64, 4, 2)
    step = step_of(model, ids_of(300, 200), torch.tensor([0, 300], device="cuda", dtype=torch.int32))
    want = step()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        got = step()
    here = step()
    torch.cuda.synchronize()
    for a, b, c in zip(got, want, here):
        assert torch.equal(a, b) and torch.equal(b, c)


@pytest.mark.parametrize("T", [0, 1])
def test_no_tokens_and_one(T):
    torch.manual_seed(T)
    model = experts.TokenModel(20, 64, 32, 4, 2)
    logits, balance = model(ids_of(T, 20, 0, 0), torch.tensor([0, T], device="cuda", dtype=torch.int32))
    (logits.float().square().sum() + balance).backward()
    assert logits.shape == (T, 20)
    for p in model.parameters():
        assert torch.isfinite(p.grad).all() and (T or (p.grad == 0).all())


def test_serving_in_8_bits_is_the_layer_in_8_bits():
    torch.manual_seed(5)
    layer = experts.ExpertLayer(200, 72, 4, 2, eight_bits=True)
    for tokens in (1, 33):
        x = torch.randn(tokens, 200, device="cuda").bfloat16()
        layer.served = None
        want = layer.serve(x)
        layer.quantise(bits=8)
        assert torch.equal(layer.serve(x), want)


def test_training_tokens_runs():
    assert all(loss == loss for loss in experts.train_tokens(steps=3))
