"""Products of floats over long inner dimensions: how the error grows.  Each addition to a running sum rounds it by 2^-24 of itself at
most; over a chain of n additions of values of either sign the sum grows as the square root of their number, and the error's
root mean square is at most 2^-24 * sqrt(n / 2) of the result's.  The bounds count the additions that are made one after the other:
   the instruction for floats   runs of 512 values, then the totals of a wavefront's runs, then eight wavefronts' totals
   parts of 16 bits             a chain of a sum for every 32 values; within those 32, and for what is left out, a few units
A sum of all values one after the other has sqrt(n / 2) with n the whole inner dimension."""
import math

import pytest
import torch

from paper_2209_02882_amd import binding

pytestmark = pytest.mark.gpu

UNIT = 2.0**-24


def by_runs(n, waves):
    return UNIT * math.sqrt(512 / 2 + n / 512 / waves / 2 + 8)


def by_parts(n):
    return UNIT * math.sqrt(n / 32 / 2 + 8)


def off(got, want):
    return float((got.double() - want).square().mean().sqrt() / want.square().mean().sqrt())


def normal(seed, *shape):
    return torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")


def some(n):
    return torch.arange(0, n, max(1, n // 64), device="cuda")


def product_off(R, K, N, layout):
    X, W = normal(1, R, K), normal(2, *((1, N, K) if layout == "nk" else (1, K, N)))
    Y = torch.empty(R, N, device="cuda")
    binding.sgap_grouped_mm(1, R, K, N, None, X, W, Y, layout)
    w = W[0].t().contiguous() if layout == "nk" else W[0]
    return off(Y[some(R)], torch.mm(X[some(R)].double(), w.double()))


def gradient_off(R, K, N, layout):
    X, dY = normal(1, R, K), normal(2, R, N)
    dW = torch.empty((1, N, K) if layout == "nk" else (1, K, N), device="cuda")
    binding.sgap_grouped_mm_wgrad(1, R, K, N, None, X, dY, dW, layout)
    got = dW[0] if layout == "nk" else dW[0].t()
    return off(got[some(N)], torch.mm(dY[:, some(N)].double().t().contiguous(), X.double()))


# few rows or columns: wavefronts share the inner dimension; 16 rows and more, 16 to 64 columns to a workgroup
@pytest.mark.parametrize("layout", ["nk", "kn"])
@pytest.mark.parametrize("R,K,N", [(1, 262_144, 64), (16, 262_144, 128), (64, 262_144, 128), (128, 65_536, 4_096), (8, 65_536, 8_192)])
def test_few_rows_by_long_weights(R, K, N, layout):
    assert product_off(R, K, N, layout) <= by_runs(K, 8)


# few weights: wavefronts share the rows, 32 x 32 and 64 x 64 weights to a workgroup
@pytest.mark.parametrize("layout", ["nk", "kn"])
@pytest.mark.parametrize("R,K,N", [(262_144, 128, 128), (262_144, 512, 256), (131_072, 1_024, 1_024)])
def test_gradient_of_few_weights_from_many_rows(R, K, N, layout):
    assert gradient_off(R, K, N, layout) <= by_runs(R, 8)


# rows at addresses that are no multiples of 16 bytes
@pytest.mark.parametrize("layout", ["nk", "kn"])
def test_rows_at_odd_addresses(layout):
    assert product_off(300, 65_533, 515, layout) <= by_runs(65_533, 1)
    assert gradient_off(65_533, 259, 131, layout) <= by_runs(65_533, 1)


# rows, columns and weights enough for tiles: parts of 16 bits
@pytest.mark.parametrize("layout", ["nk", "kn"])
@pytest.mark.parametrize("R,K,N", [(2_048, 4_096, 2_048), (2_000, 65_536, 2_040), (4_096, 16_384, 1_024)])
def test_many_rows_by_long_weights(R, K, N, layout):
    assert product_off(R, K, N, layout) <= by_parts(K)


@pytest.mark.parametrize("layout", ["nk", "kn"])
@pytest.mark.parametrize("R,K,N", [(16_384, 2_048, 2_048), (65_536, 2_048, 2_048), (150_001, 1_032, 2_048)])
def test_gradient_of_many_weights_from_many_rows(R, K, N, layout):
    assert gradient_off(R, K, N, layout) <= by_parts(R)


# a tile with a sum that is not finite goes by the instruction for floats: its other sums are no worse for it
@pytest.mark.parametrize("layout", ["nk", "kn"])
def test_long_sums_beside_one_that_is_infinite(layout):
    R, K, N = 2_048, 65_536, 2_048
    X, W = normal(1, R, K), normal(2, *((1, N, K) if layout == "nk" else (1, K, N)))
    X[5, 7] = float("inf")
    Y = torch.empty(R, N, device="cuda")
    binding.sgap_grouped_mm(1, R, K, N, None, X, W, Y, layout)
    w = W[0].t().contiguous() if layout == "nk" else W[0]
    assert torch.isinf(Y[5]).all()
    assert off(Y[6:70], torch.mm(X[6:70].double(), w.double())) <= by_runs(K, 1)


@pytest.mark.parametrize("layout", ["nk", "kn"])
def test_long_gradients_beside_one_that_is_infinite(layout):
    R, K, N = 65_536, 2_048, 2_048
    X, dY = normal(1, R, K), normal(2, R, N)
    dY[100, 5] = float("inf")
    dW = torch.empty((1, N, K) if layout == "nk" else (1, K, N), device="cuda")
    binding.sgap_grouped_mm_wgrad(1, R, K, N, None, X, dY, dW, layout)
    got = dW[0] if layout == "nk" else dW[0].t()
    assert torch.isinf(got[5]).all()
    assert off(got[6:70], torch.mm(dY[:, 6:70].double().t().contiguous(), X.double())) <= by_runs(R, 1)
