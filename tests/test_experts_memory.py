"""Workspaces and laid-out weights have as much memory as their number of elements says: a tensor that repeats its elements, or
skips some, is refused before anything is launched."""
import pytest
import torch

from paper_2209_02882_amd import binding


class OnDevice(torch.Tensor):
    """A host tensor that says it is on the device, for the binding's own checks."""
    is_cuda = property(lambda self: True)


def make(t, device):
    return t.cuda() if device else t.as_subclass(OnDevice)


def repeated(device, size):
    """`size` elements, the same byte over and over; as many, every other one of twice the memory."""
    return [make(torch.zeros(1, dtype=torch.uint8), device).expand(size), make(torch.zeros(2 * size, dtype=torch.uint8), device)[::2]]


@pytest.mark.parametrize("device", [False, pytest.param(True, marks=pytest.mark.gpu)])
def test_weights_and_workspaces_that_are_not_contiguous(device):
    G, K, N, R = 1, 128, 16, 4
    size = binding.sgap_w4_layout_size(G, K, N, 64)
    half = lambda *shape: make(torch.zeros(shape, dtype=torch.float16), device)  # noqa: E731
    codes, scales = make(torch.zeros(G, N, K // 2, dtype=torch.uint8), device), half(G, N, K // 64)
    for weights in repeated(device, size):
        with pytest.raises(ValueError, match="weights must be contiguous"):
            binding.sgap_w4_layout(G, K, N, 64, codes, scales, None, weights)
        with pytest.raises(ValueError, match="weights must be contiguous"):
            binding.sgap_grouped_mm_w4(G, R, K, N, 64, None, half(R, K), weights, half(R, N))
    T, E, k = 100, 8, 2
    i32 = lambda *shape: make(torch.zeros(shape, dtype=torch.int32), device)  # noqa: E731
    f32 = lambda *shape: make(torch.zeros(shape), device)  # noqa: E731
    for workspace in repeated(device, binding.sgap_route_topk_workspace_size(T, E, k)):
        with pytest.raises(ValueError, match="workspace must be contiguous"):
            binding.sgap_route_topk(T, E, k, f32(T, E), f32(T, k), i32(T, k), i32(T, k), i32(T * k), i32(E + 1), workspace=workspace)
