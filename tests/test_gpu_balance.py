"""The router's balance loss, its counts and its gradient, against plain forms in 64 bits."""
import numpy as np
import pytest
import torch

from experts_util import E as EPS
from experts_util import assert_within, offsets_of, random, route
from paper_2209_02882_amd import binding
from tokens_util import balance, filled

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.float16, torch.bfloat16]


def chosen(logits, k):
    """What the router leaves: the k largest, -1 where only -infinity is left."""
    top, experts = torch.sort(logits.double(), dim=1, descending=True, stable=True)
    return torch.where(top[:, :k] > float("-inf"), experts[:, :k], torch.full_like(experts[:, :k], -1)).int().contiguous()


def workspace(T, E, k, S):
    return torch.full((binding.sgap_route_balance_workspace_size(T, E, k, S),), 0x7f, dtype=torch.uint8, device="cuda")


def forward(logits, experts, segments, k):
    T, E = logits.shape
    S = 1 if segments is None else len(segments) - 1
    loss, counts, rows = filled(torch.float32, 1), filled(torch.int32, S, E), filled(torch.int32, S)
    binding.sgap_route_balance(T, E, k, S, logits, experts, segments, loss, counts, rows, workspace=workspace(T, E, k, S))
    return loss, counts, rows


def gradient(logits, experts, segments, k, counts, rows, dloss=1.0, dlogits=None, **more):
    T, E = logits.shape
    S = 1 if segments is None else len(segments) - 1
    dlogits = torch.full_like(logits, float("nan")) if dlogits is None else dlogits
    binding.sgap_route_balance_grad(T, E, k, S, logits, experts, segments, counts, rows, torch.full((1,), dloss, device="cuda"), dlogits, **more)
    return dlogits


def check(logits, k, segments=None, experts=None, dloss=1.0):
    T, E = logits.shape
    experts = chosen(logits, k) if experts is None else experts
    on = None if segments is None else segments.cuda()
    got = forward(logits.cuda(), experts.cuda(), on, k)
    loss, counts, rows, grad, size = balance(logits, experts, segments, k)
    np.testing.assert_array_equal(got[1].cpu().numpy(), counts)
    np.testing.assert_array_equal(got[2].cpu().numpy(), rows)
    # a logit less the largest is rounded (its size times 2^-24), exp and the division by E summed values each, then sums of T; all
    # in units of 2^-23
    real = torch.where(torch.isfinite(logits), logits.double(), torch.zeros(1, dtype=torch.float64))
    wide = float(real.max() - real.min()) if T else 0.0
    assert_within(got[0], np.array([loss]), (T + E + wide + 16) * EPS * max(abs(loss), 1e-300), "loss")
    dlogits = gradient(logits.cuda(), experts.cuda(), on, k, got[1], got[2], dloss)
    assert_within(dlogits, dloss * grad, (2 * E + 2 * wide + 24) * EPS * abs(dloss) * size, "gradient")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,E,k", [(1, 1, 1), (1, 8, 2), (2, 7, 7), (63, 16, 1), (64, 17, 4), (65, 60, 6), (200, 128, 8), (130, 200, 5), (300, 256, 16),
                                   (70, 257, 3), (100, 513, 9), (90, 1000, 16), (33, 1024, 2), (5000, 12, 3)])
def test_loss_and_gradient(T, E, k, dtype):
    check((random(T + E, T, E, scale=2.0) + random(E, E)).to(dtype), k, dloss=0.25)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("sizes", [[0], [5], [0, 64, 0, 65, 1, 0], [1] * 90, [200, 0, 0, 31], [0] * 70 + [3]])
def test_sequences(sizes, dtype):
    segments = offsets_of(sizes)
    T = sum(sizes) + 7  # some tokens behind the last sequence
    check((random(T, T, 20) + random(1, 20)).to(dtype), 3, segments)


# as many sequences as share the compute units by smaller workgroups and one less, many of them empty or of one token, and a long one; more
# than one, two and three rounds of a search in 64 places; more experts than a smaller workgroup has
@pytest.mark.parametrize("S,E", [(64, 9), (65, 9), (511, 20), (512, 20), (700, 300), (1_000, 1_024), (4_097, 17), (65_536, 3)])
def test_many_sequences(S, E):
    sizes = np.random.default_rng(S).choice([0, 0, 1, 1, 2, 3], S)
    sizes[S // 3], sizes[-1] = 300, 2
    segments = offsets_of(sizes.tolist()) + 5  # some tokens before the first sequence, some behind the last
    check((random(S, int(sizes.sum()) + 12, E) + random(1, E)).to(torch.bfloat16), 2, segments)


def test_tokens_before_the_first_sequence():
    check(random(1, 100, 9), 2, torch.tensor([13, 50, 50, 90], dtype=torch.int32))


@pytest.mark.parametrize("lowest", [float("-inf"), None])
def test_masks(lowest):
    T, E, k = 150, 40, 4
    for dtype in TYPES:
        x = random(3, T, E, scale=1.5)
        low = torch.finfo(dtype).min if lowest is None else lowest
        x[torch.rand(T, E, generator=torch.Generator().manual_seed(1)) < 0.4] = low
        x[::7] = low                 # nothing left (or, of the lowest value, all alike)
        x[3::11, 1:] = low           # one expert left
        check_masked = x.to(dtype)
        experts = chosen(check_masked, k)
        on = check_masked.cuda(), experts.cuda()
        loss, counts, rows = forward(*on, None, k)
        want, c, n, grad, size = balance(check_masked, experts, None, k)
        np.testing.assert_array_equal(counts.cpu().numpy(), c)
        np.testing.assert_array_equal(rows.cpu().numpy(), n)
        # differences of 6 in what is left of a row, so 32 with the sums of 40 values and 150 tokens
        assert_within(loss, np.array([want]), (T + E + 32) * EPS * want)
        dlogits = gradient(*on, None, k, counts, rows)
        assert_within(dlogits, grad, (2 * E + 64) * EPS * size)
        if lowest is not None:
            assert not dlogits[::7].any()


def test_padding_has_no_part_whatever_its_logits():
    # tokens whose choices somebody took away: NaN in their logits is not looked at
    x = random(1, 90, 12)
    experts = chosen(x, 2)
    experts[::5] = -1
    experts[1::5, 1] = 12    # one choice outside the experts
    want = balance(x, experts, None, 2)
    x[::5] = float("nan")
    loss, counts, rows = forward(x.cuda(), experts.cuda(), None, 2)
    assert_within(loss, np.array([want[0]]), 130 * EPS * want[0])
    np.testing.assert_array_equal(counts.cpu().numpy(), want[1])
    np.testing.assert_array_equal(rows.cpu().numpy(), want[2])
    dlogits = gradient(x.cuda(), experts.cuda(), None, 2, counts, rows)
    assert_within(dlogits, want[3], 60 * EPS * want[4])


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_a_token_that_is_no_number_is_seen_in_the_loss_and_its_own_gradient(bad):
    x = random(1, 80, 12)
    x[17, 3] = bad
    experts = chosen(torch.where(torch.isfinite(x), x, torch.full_like(x, 9.0)), 2)
    loss, counts, rows = forward(x.cuda(), experts.cuda(), None, 2)
    assert torch.isnan(loss).all() and int(rows) == 80
    dlogits = gradient(x.cuda(), experts.cuda(), None, 2, counts, rows)
    assert torch.isnan(dlogits[17]).all()
    assert torch.isfinite(dlogits[:17]).all() and torch.isfinite(dlogits[18:]).all()


def test_an_even_load_has_loss_one_and_no_gradient():
    E, k = 8, 2
    experts = torch.stack([torch.arange(64) % E, (torch.arange(64) + 1) % E], dim=1).int()
    x = random(1, 64, E).cuda()
    loss, counts, rows = forward(x, experts.cuda(), None, k)
    assert torch.equal(counts, torch.full_like(counts, 16))
    assert abs(loss.item() - 1) <= 80 * EPS
    assert not gradient(x, experts.cuda(), None, k, counts, rows).any()


def test_near_an_even_load_the_gradient_keeps_its_digits():
    # 2^19 tokens' counts but for one pair even: f is within 2^-18 of one, and the gradient is made of what is beyond
    T, E, k = 3 * 2**17, 3, 1
    x, experts = random(1, 48, E), (torch.arange(T) % E).int()
    experts[0] = 1
    counts = torch.bincount(experts.long(), minlength=E).int()
    rows = torch.tensor([T], dtype=torch.int32)
    dlogits = gradient(x.cuda(), experts[:48].view(48, 1).contiguous().cuda(), None, k, counts.cuda(), rows.cuda())
    p = torch.softmax(x.double(), dim=1)
    f1 = (counts.double() * E - T) / T
    want, size = p * (f1 - (p @ f1)[:, None]) / T, p * (f1.abs() + (p @ f1.abs())[:, None]) / T
    assert_within(dlogits, want, 50 * EPS * size)


@pytest.mark.parametrize("dtype", TYPES)
def test_the_gradient_is_added(dtype):
    segments = offsets_of([40, 0, 23])
    x, was = random(1, 70, 18).to(dtype), random(2, 70, 18, scale=0.01).to(dtype)
    experts = chosen(x, 3)
    loss, counts, rows = forward(x.cuda(), experts.cuda(), segments.cuda(), 3)
    got = gradient(x.cuda(), experts.cuda(), segments.cuda(), 3, counts, rows, 0.5, was.cuda(), accumulate=True)
    _, _, _, grad, size = balance(x, experts, segments, 3)
    assert torch.equal(got[63:].cpu(), was[63:])
    assert_within(got, was.double().numpy() + 0.5 * grad, 90 * EPS * (size + np.abs(was.double().numpy())))


@pytest.mark.parametrize("E", [17, 60, 300])
def test_rows_apart(E):
    x = random(1, 50, E + 9)
    part = x[:, 4:4 + E]
    experts = chosen(part, 2)
    on, out = x.cuda(), filled(torch.float32, 50, E + 3)
    loss, counts, rows = forward(on[:, 4:4 + E], experts.cuda(), None, 2)
    gradient(on[:, 4:4 + E], experts.cuda(), None, 2, counts, rows, dlogits=out[:, 1:1 + E])
    want = balance(part, experts, None, 2)
    assert_within(loss, np.array([want[0]]), (E + 90) * EPS * want[0])
    assert_within(out[:, 1:1 + E].contiguous(), want[3], (2 * E + 50) * EPS * want[4])
    assert torch.isnan(out[:, 0]).all() and torch.isnan(out[:, 1 + E:]).all()


def test_gradient_against_differences():
    # with the counts held, the loss is smooth: central differences of its 64-bit form with h = 2^-10 are off by h^2 / 6 times a third
    # derivative, which p's bound by 1 keeps under 12 |f|
    x, k, h = random(1, 24, 10), 2, 2.0**-10
    experts = chosen(x, k)
    _, counts, rows = forward(x.cuda(), experts.cuda(), None, k)
    got = gradient(x.cuda(), experts.cuda(), None, k, counts, rows).double().cpu()
    f = torch.from_numpy(balance(x, experts, None, k)[1]).double() * 10 / (k * 24)

    def loss(z):
        return (torch.softmax(z, dim=1).mean(0) * f).sum()

    for t, e in [(0, 0), (5, 9), (23, 4)]:
        step = torch.zeros(24, 10, dtype=torch.float64)
        step[t, e] = h
        slope = (loss(x.double() + step) - loss(x.double() - step)) / (2 * h)
        assert abs(got[t, e] - slope) <= 2 * h * h * f.max() / 24 + 50 * EPS * f.max() / 24


def test_after_the_router_and_captured():
    T, E, k = 700, 48, 4
    x = random(1, T, E).cuda()
    segments = offsets_of([300, 0, 380]).cuda()
    gates, experts, slot = filled(torch.float32, T, k), filled(torch.int32, T, k), filled(torch.int32, T, k)
    order, offsets = filled(torch.int32, T * k), filled(torch.int32, E + 1)
    route_ws = torch.empty(binding.sgap_route_topk_workspace_size(T, E, k), dtype=torch.uint8, device="cuda")
    loss, counts, rows = filled(torch.float32, 1), filled(torch.int32, 3, E), filled(torch.int32, 3)
    ws, dlogits, dloss = workspace(T, E, k, 3), torch.empty_like(x), torch.ones(1, device="cuda")

    def step():
        binding.sgap_route_topk(T, E, k, x, gates, experts, slot, order, offsets, workspace=route_ws)
        binding.sgap_route_balance(T, E, k, 3, x, experts, segments, loss, counts, rows, workspace=ws)
        binding.sgap_route_topk_grad(T, E, k, x, gates, experts, gates, dlogits)
        binding.sgap_route_balance_grad(T, E, k, 3, x, experts, segments, counts, rows, dloss, dlogits, accumulate=True)

    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in (2, 3, 4):
        x.copy_(random(seed, T, E))
        for t in (loss, dlogits):
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        host = x.cpu()
        want = balance(host, torch.from_numpy(route(host, k, True)[1]), segments.cpu(), k)
        assert_within(loss, np.array([want[0]]), (T + E + 30) * EPS * want[0])
        np.testing.assert_array_equal(counts.cpu().numpy(), want[1])
        alone = torch.empty_like(x)
        binding.sgap_route_topk_grad(T, E, k, x, gates, experts, gates, alone)
        assert_within(dlogits, alone.double().cpu().numpy() + want[3], 200 * EPS * (want[4] + alone.double().abs().cpu().numpy()))


def test_the_same_bits_on_every_call_and_on_two_streams():
    x = random(1, 9000, 64, dtype=torch.bfloat16).cuda()
    experts = chosen(x.cpu(), 6).cuda()
    first = forward(x, experts, None, 6)
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    again = []
    for s in streams * 2:
        with torch.cuda.stream(s):
            again.append(forward(x, experts, None, 6))
    torch.cuda.synchronize()
    for got in again:
        assert all(torch.equal(a, b) for a, b in zip(got, first))


def test_segments_in_no_order_touch_nothing_else():
    # (what they give is nothing that the header promises; all of it stays inside the arrays)
    T, E, k = 500, 16, 2
    x = random(1, T, E).cuda()
    experts = chosen(x.cpu(), k).cuda()
    for list_ in ([900, -5, 300, 100], [0, 500, 0, 500], [-2**31, 2**31 - 1, 7, 7]):
        segments = torch.tensor(list_, dtype=torch.int32, device="cuda")
        loss, counts, rows = forward(x, experts, segments, k)
        dlogits = gradient(x, experts, segments, k, counts, rows)
        assert not torch.isnan(dlogits).any() and (counts >= 0).all()


def test_a_short_workspace_is_refused():
    x, i = torch.zeros(9, 4, device="cuda"), torch.zeros(9, 2, dtype=torch.int32, device="cuda")
    with pytest.raises(binding.SgapError, match="workspace"):
        binding.sgap_route_balance(9, 4, 2, 1, x, i, None, torch.zeros(1, device="cuda"), i[:2].clone(), i[0, :1].clone())
    with pytest.raises(ValueError, match="segments"):
        binding.sgap_route_balance(9, 4, 2, 2, x, i, i[0].clone(), torch.zeros(1, device="cuda"), i[:4].clone(), i[0].clone())
