"""The router and the way back against plain 64-bit forms: every number of experts per lane, ties, masks that leave few or no
experts, values that are no numbers, one token to many blocks of them."""
import numpy as np
import pytest
import torch

from experts_util import E, assert_within, random, route, route_grad
from paper_2209_02882_amd import binding

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.float16, torch.bfloat16]


def run_route(logits, k, renormalise, stream=None):
    T, n = logits.shape
    i32 = dict(dtype=torch.int32, device="cuda")
    gates = torch.full((T, k), float("nan"), device="cuda")
    experts, slot = (torch.full((T, k), -7, **i32) for _ in range(2))
    order, offsets = torch.full((T * k,), -7, **i32), torch.full((n + 1,), -7, **i32)
    size = binding.sgap_route_topk_workspace_size(T, n, k)
    workspace = torch.full((size,), 0x5a, dtype=torch.uint8, device="cuda") if size else None
    binding.sgap_route_topk(T, n, k, logits, gates, experts, slot, order, offsets, renormalise, workspace)
    return gates, experts, slot, order, offsets


def check_route(logits, k, renormalise, what):
    got = run_route(logits.cuda(), k, renormalise)
    want = route(logits, k, renormalise)
    for name, g, w in zip(("experts", "slot", "order", "offsets"), got[1:], want[1:]):
        np.testing.assert_array_equal(g.cpu().numpy(), w, err_msg=f"{what}: {name}")
    # exp of a difference that is rounded (up to 2^-24 * 88 of it) and good to two units, and a sum of n of them
    slack = np.abs(want[0]) * (logits.shape[1] + 200) * E + 1e-37
    assert_within(got[0], want[0], np.nan_to_num(slack), f"{what}: gates")
    return got, want


def check_grad(logits, got, k, renormalise, what):
    T, n = logits.shape
    dgates = random(99, T, k)
    dlogits = torch.full((T, n), float("nan"), dtype=logits.dtype, device="cuda")
    binding.sgap_route_topk_grad(T, n, k, logits.cuda(), got[0], got[1], dgates.cuda(), dlogits, renormalise)
    gates, experts = got[0].double().cpu().numpy(), got[1].cpu().numpy()
    want, size = route_grad(logits, gates, experts, dgates.double().numpy(), renormalise)
    assert_within(dlogits, want, size * (n + k + 200) * E + 1e-37, f"{what}: dlogits")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,n,k", [(1, 1, 1), (1, 8, 2), (4, 64, 4), (63, 17, 3), (64, 16, 16), (65, 33, 5), (130, 60, 6), (300, 128, 8),
                                   (257, 129, 7), (500, 256, 16), (70, 257, 1), (200, 512, 10), (129, 513, 16), (3, 1024, 16),
                                   (1000, 1000, 2)])
def test_choice_lists_and_gradient(T, n, k, dtype):
    for renormalise in (True, False):
        logits = random(T * 7 + n, T, n, dtype=dtype, scale=2.0)
        what = f"{T} tokens, {n} experts, k {k}, {dtype}, renormalise {renormalise}"
        got, _ = check_route(logits, k, renormalise, what)
        check_grad(logits, got, k, renormalise, what)


@pytest.mark.parametrize("T", [40, 400])
@pytest.mark.parametrize("dtype", TYPES)
def test_ties_go_to_the_lowest_expert(T, dtype):
    gen = torch.Generator().manual_seed(5)
    logits = torch.randint(-1, 2, (T, 90), generator=gen).to(dtype)  # three values only
    logits[3] = 0.0
    logits[4, ::2], logits[4, 1::2] = 0.0, -0.0
    got, _ = check_route(logits, 7, True, "ties")
    assert got[1][3].tolist() == list(range(7)) and got[1][4].tolist() == list(range(7))


@pytest.mark.parametrize("T,n,k", [(50, 20, 4), (700, 200, 8), (90, 700, 3)])
@pytest.mark.parametrize("renormalise", [True, False])
def test_masks_that_leave_few_experts_or_none(T, n, k, renormalise):
    logits = random(11, T, n, dtype=torch.bfloat16)
    gen = torch.Generator().manual_seed(6)
    logits[torch.rand(T, n, generator=gen) < 0.4] = float("-inf")
    logits[0] = float("-inf")
    logits[T - 1] = float("-inf")
    logits[5, :] = float("-inf")
    logits[5, n - 1] = 1.0
    logits[6] = torch.finfo(torch.bfloat16).min
    logits[7, 1:] = torch.finfo(torch.bfloat16).min
    got, want = check_route(logits, k, renormalise, "masks")
    assert want[1][0].tolist() == [-1] * k and (got[0][0] == 0).all()
    assert want[1][5].tolist() == [n - 1] + [-1] * (k - 1)
    check_grad(logits, got, k, renormalise, "masks")
    # every token without an expert
    logits[:] = float("-inf")
    got, _ = check_route(logits, k, renormalise, "nothing left")
    assert int(got[4].abs().sum()) == 0 and (got[3] == -1).all()
    check_grad(logits, got, k, renormalise, "nothing left")


@pytest.mark.parametrize("renormalise", [True, False])
def test_values_that_are_no_numbers(renormalise):
    logits = random(12, 30, 40)
    logits[1, 7] = float("nan")
    logits[2, [3, 9]] = float("nan")
    logits[3, 5] = float("inf")
    logits[4, [5, 6]] = float("inf")
    logits[5, 4], logits[5, 30] = float("inf"), float("nan")
    logits[6] = float("nan")
    got, want = check_route(logits, 3, renormalise, "no numbers")
    assert torch.isnan(got[0][1:7]).all() and want[1][1, 0] == 7 and want[1][2, :2].tolist() == [3, 9]
    assert torch.isfinite(got[0][7:]).all()


def test_rows_apart_and_many_tokens():
    wide = random(13, 5000, 97, dtype=torch.float16)
    logits = wide[:, 5:70]  # rows of 65, 97 apart, not aligned
    T, n, k = 5000, 65, 4
    dev = wide.cuda()[:, 5:70]
    got = run_route(dev, k, False)
    want = route(logits, k, False)
    for g, w in zip(got[1:], want[1:]):
        np.testing.assert_array_equal(g.cpu().numpy(), w)
    dgates = random(14, T, k)
    out = torch.full((T, 80), 3.0, dtype=torch.float16, device="cuda")
    binding.sgap_route_topk_grad(T, n, k, dev, got[0], got[1], dgates.cuda(), out[:, 8:73], False)
    ref, size = route_grad(logits, got[0].double().cpu().numpy(), got[1].cpu().numpy(), dgates.double().numpy(), False)
    assert_within(out[:, 8:73], ref, size * 300 * E + 1e-37, "strided dlogits")
    assert (out[:, :8] == 3).all() and (out[:, 73:] == 3).all()


def test_no_tokens():
    got = run_route(torch.empty(0, 12, device="cuda"), 3, True)
    assert got[4].tolist() == [0] * 13


@pytest.mark.parametrize("renormalise", [True, False])
def test_gradient_against_differences(renormalise):
    T, n, k, h = 20, 24, 4, 2.0**-6
    logits, dgates, step = random(15, T, n), random(16, T, k), random(17, T, n)
    # choices far enough apart that the step does not change them
    logits = (torch.argsort(torch.argsort(logits, dim=1), dim=1).float() - n / 2) * 0.25
    got = run_route(logits.cuda(), k, renormalise)
    dlogits = torch.empty(T, n, device="cuda")
    binding.sgap_route_topk_grad(T, n, k, logits.cuda(), got[0], got[1], dgates.cuda(), dlogits, renormalise)
    step = step.clamp(-2, 2)
    up, down = run_route((logits + h * step).cuda(), k, renormalise), run_route((logits - h * step).cuda(), k, renormalise)
    assert torch.equal(up[1], got[1]) and torch.equal(down[1], got[1])
    slope = ((up[0] - down[0]).double().cpu() / (2 * h) * dgates.double()).sum(dim=1)
    exact = (dlogits.double().cpu() * step.double()).sum(dim=1)
    # third derivative of a softmax along a step of at most 2: under 8 * 2^3 / 6 * h^2 a gate; rounding: 2^-21 / h
    bound = dgates.abs().double().sum(dim=1) * (11 * h * h + 2.0**-21 / h)
    assert ((slope - exact).abs() <= bound).all()


def combine_reference(Z, slot, gates):
    T, k = slot.shape
    z = torch.cat([Z.double(), torch.zeros(1, Z.shape[1], dtype=torch.float64)])[slot.long()]  # -1: the row of zeros
    g = torch.ones(T, k, dtype=torch.float64) if gates is None else gates.double()
    return (z * g[..., None]).sum(1), (z.abs() * g.abs()[..., None]).sum(1), z


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,k,D", [(1, 1, 1), (3, 2, 5), (1, 16, 7), (13, 2, 1001), (5, 4, 8), (64, 3, 64), (33, 8, 513), (4, 6, 4099),
                                   (100, 9, 96), (4100, 2, 40), (7, 2, 2048), (1030, 5, 130)])
def test_combine_and_its_gradients(T, k, D, dtype):
    R = T * k
    Z, gates, dout = random(T + D, R, D, dtype=dtype), random(3, T, k), random(4, T, D, dtype=dtype)
    gen = torch.Generator().manual_seed(T * D)
    order = torch.randperm(R, generator=gen).int()
    missing = torch.rand(R, generator=gen) < 0.2  # pairs without a place: their places lie at the end
    kept = order[~missing[order.long()]]
    order = torch.cat([kept, torch.full((R - kept.numel(),), -1, dtype=torch.int32)])
    slot = torch.full((R,), -1, dtype=torch.int32)
    slot[kept.long()] = torch.arange(kept.numel(), dtype=torch.int32)
    slot = slot.view(T, k)
    dev = [t.cuda() for t in (Z, slot, order, gates, dout)]
    for g in (gates, None):
        out = torch.full((T, D), float("nan"), dtype=dtype, device="cuda")
        binding.sgap_route_combine(T, k, D, dev[0], dev[1], None if g is None else dev[3], out)
        want, size, z = combine_reference(Z, slot, g)
        assert_within(out, want, size * (k + 4) * E, f"combine {T} {k} {D} {dtype} gates {g is not None}")
    dZ = torch.full((R, D), float("nan"), dtype=dtype, device="cuda")
    dgates = torch.full((T, k), float("nan"), device="cuda")
    binding.sgap_route_combine_grad(T, k, D, *dev[:2], dev[2], dev[3], dev[4], dZ, dgates)
    want = torch.zeros(R, D, dtype=torch.float64)
    want[:kept.numel()] = gates.double().view(-1)[kept.long()][:, None] * dout.double()[torch.div(kept.long(), k, rounding_mode="floor")]
    assert_within(dZ, want, want.abs() * E, "dZ")
    d = dout.double()[:, None, :]
    assert_within(dgates, (z * d).sum(2), (z * d).abs().sum(2) * (D + 4) * E, "dgates")


def test_combine_passes_infinities_on():
    Z = torch.ones(4, 24)
    Z[2, 5], Z[3, 6] = float("inf"), float("nan")
    slot = torch.tensor([[0, 1], [2, 3]], dtype=torch.int32)
    gates = torch.tensor([[0.5, 0.5], [0.25, 0.0]])
    out = torch.empty(2, 24, device="cuda")
    binding.sgap_route_combine(2, 2, 24, Z.cuda(), slot.cuda(), gates.cuda(), out)
    assert torch.equal(out[0].cpu(), torch.ones(24))
    row = out[1].cpu()
    assert row[5] == float("inf") and torch.isnan(row[6]) and torch.isfinite(row[7:]).all()
