"""Calls of more workgroups than a launch may have threads for (2^32 of them): they go out as several launches.  Small values, whose
sums are exact in every type."""
import pytest
import torch

from paper_2209_02882_amd import binding

pytestmark = pytest.mark.gpu


def small(seed, *shape, dtype=torch.bfloat16):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(-3, 4, shape, generator=gen, device="cuda", dtype=torch.int8).to(dtype)


def test_sums_back_of_many_tokens():
    T, D = 2**26 + 5, 8
    Z = small(1, T, D)
    slot = torch.arange(T - 1, -1, -1, dtype=torch.int32, device="cuda")  # its own inverse
    gates = torch.full((T, 1), 2.0, device="cuda")
    out = torch.full_like(Z, float("nan"))
    binding.sgap_route_combine(T, 1, D, Z, slot, gates, out)
    assert torch.equal(out, 2 * Z.flip(0))
    dZ, dgates = torch.full_like(Z, float("nan")), torch.full_like(gates, float("nan"))
    binding.sgap_route_combine_grad(T, 1, D, Z, slot, slot, gates, out, dZ, dgates)
    assert torch.equal(dZ, 2 * out.flip(0))
    assert torch.equal(dgates[:, 0], (Z.flip(0).float() * out.float()).sum(1))


def test_sums_back_of_rows_of_one_value():
    T = 2**26 + 3
    Z, slot = small(2, T, 1), torch.arange(T, dtype=torch.int32, device="cuda")
    slot[-1] = -1
    out = torch.full_like(Z, float("nan"))
    binding.sgap_route_combine(T, 1, 1, Z, slot, None, out)
    Z[-1] = 0
    assert torch.equal(out, Z)


def test_many_tokens_choose():
    T, n = 2**28 + 7, 2
    logits = small(3, T, n)
    i32 = dict(dtype=torch.int32, device="cuda")
    gates = torch.full((T, 1), float("nan"), device="cuda")
    experts, slot, order = (torch.full((T,), -7, **i32) for _ in range(3))
    offsets = torch.full((n + 1,), -7, **i32)
    workspace = torch.empty(binding.sgap_route_topk_workspace_size(T, n, 1), dtype=torch.uint8, device="cuda")
    binding.sgap_route_topk(T, n, 1, logits, gates, experts, slot, order, offsets, renormalise=False, workspace=workspace)
    chosen = logits[:, 1] > logits[:, 0]
    assert torch.equal(experts, chosen.int())
    first = int(T - chosen.sum())
    assert offsets.tolist() == [0, first, T]
    assert torch.equal(order[:first], (~chosen).nonzero()[:, 0].int()) and torch.equal(order[first:], chosen.nonzero()[:, 0].int())
    slot[order.long()] -= torch.arange(T, **i32)
    assert not slot.any()
    # gates and their gradient: the probability of the larger logit, and p (1 - p)
    p = torch.sigmoid((logits[:, 0] - logits[:, 1]).abs().float())
    assert (gates[:, 0] - p).abs().max() <= 2.0**-20
    dlogits = torch.full_like(logits, float("nan"))
    binding.sgap_route_topk_grad(T, n, 1, logits, gates, experts, torch.ones_like(gates), dlogits, renormalise=False)
    p *= 1 - p
    sign = 1 - 2 * chosen.int()
    assert (dlogits[:, 0] - sign * p).abs().max() <= 2.0**-10 and (dlogits[:, 1] + sign * p).abs().max() <= 2.0**-10


def test_rows_and_columns_of_one_value():
    R = 2**29 + 40  # 32 rows to a tile
    X = small(4, R, 1, dtype=torch.float16)
    Y = torch.full_like(X, float("nan"))
    binding.sgap_grouped_mm(1, R, 1, 1, None, X, torch.full((1, 1, 1), 3.0, dtype=torch.float16, device="cuda"), Y)
    assert torch.equal(Y, 3 * X)


def test_gradients_of_many_groups():
    # 17 tiles of columns to each of 2^20 groups, the last of which has all rows
    G, K, N, R = 2**20, 1, 2100, 5
    offsets = torch.zeros(G + 1, dtype=torch.int32, device="cuda")
    offsets[-1] = R
    X, dY = small(5, R, K), small(6, R, N)
    dW = torch.full((G, N, K), float("nan"), dtype=X.dtype, device="cuda")
    binding.sgap_grouped_mm_wgrad(G, R, K, N, offsets, X, dY, dW)
    assert torch.equal(dW[-1].float(), (dY.float().t().contiguous() @ X.float())) and not dW[:-1].any()


def test_4_bit_products_of_many_groups_without_inner_values():
    G, N, R = 2**20, 2**16, 3
    Y = torch.full((R, N), float("nan"), dtype=torch.bfloat16, device="cuda")
    offsets = torch.zeros(G + 1, dtype=torch.int32, device="cuda")
    weights = torch.empty(binding.sgap_w4_layout_size(G, 0, N, 64), dtype=torch.uint8, device="cuda")
    binding.sgap_grouped_mm_w4(G, R, 0, N, 64, offsets, torch.empty(R, 0, dtype=torch.bfloat16, device="cuda"), weights, Y)
    assert not Y.any()
