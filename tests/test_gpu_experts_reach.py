"""Products over groups sized by the rule that picks the kernel, which each test asks first: tiles loaded past the registers with X
beyond 4 GiB, with workgroups that begin at different places, with floats at the ends of their range and values that are no
numbers; and instances that ordinary sizes do not take."""
import numpy as np
import pytest
import torch

from experts_plan import BEYOND_4_GIB, FEW, TILES, plan
from experts_util import E, assert_within, grouped_mm, grouped_wgrad, offsets_of, random
from paper_2209_02882_amd import binding
from test_gpu_experts_products import OTHER, check, result

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
TYPES = [F32, F16, BF16]


def weights(seed, G, K, N, dtype, layout, scale=None):
    return random(seed, *((G, N, K) if layout == "nk" else (G, K, N)), dtype=dtype, scale=K**-0.5 if scale is None else scale)


# --------------------------------------------------------------------------
# X beyond 4 GiB
# --------------------------------------------------------------------------

@pytest.mark.parametrize("layout", ["nk", "kn"])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("sizes,K,N", BEYOND_4_GIB)
def test_rows_beyond_4_gib(sizes, K, N, dtype, layout):
    G, R, ld, x_rows = len(sizes), sum(sizes), (1 << 16) + 8, 36_000 if dtype != F32 else 18_000
    flat = torch.empty(x_rows * ld, dtype=dtype, device="cuda")
    X = flat.view(x_rows, ld)[:, :K]
    X.normal_(generator=torch.Generator(device="cuda").manual_seed(1))
    # the first rows, the last ones, and those on either side of 2, 4 and 8 GiB
    at = [0, 1, 5, x_rows - 1, x_rows - 2, 8_191, 8_192, 16_383, 16_384, 17_000]
    src = torch.tensor((at * (R // len(at) + 1))[:R], dtype=torch.int32)
    W, dY = weights(3, G, K, N, dtype, layout), random(4, R, N, dtype=dtype)
    taken = X[src.long().cuda()].cpu()
    offsets = offsets_of(sizes)
    Y, dW = result(R, N, dtype), torch.full_like(W, float("nan")).cuda()
    binding.sgap_grouped_mm(G, R, K, N, offsets.cuda(), X, W.cuda(), Y, layout, src=src.cuda())
    binding.sgap_grouped_mm_wgrad(G, R, K, N, offsets.cuda(), X, dY.cuda(), dW, layout, src=src.cuda())
    want, size = grouped_mm(offsets, taken, W, layout, R)
    assert_within(Y, want, size * (K + 4) * E)
    want, size = grouped_wgrad(offsets, taken, dY, layout)
    assert_within(dW, want, size * (max(sizes) + 4) * E)


# --------------------------------------------------------------------------
# weights that pass once, in rows of a multiple of 4,096 bytes
# --------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("row_bytes", [4_096, 12_288])
def test_workgroups_that_begin_apart(row_bytes, dtype):
    K = row_bytes // dtype.itemsize
    few = [(7 * g) % 6 for g in range(40)]
    assert plan(40, sum(few) + 3, K, 2_056, dtype, "nk").apart
    check(few, K, 2_056, dtype, "nk", k=2, extra=3, pad=8)
    more = [40 + g for g in range(12)] + [0, 64, 100, 0]
    assert plan(16, sum(more) + 70, K, 2_056, dtype, "nk").apart
    check(more, K, 2_056, dtype, "nk", extra=70)


# --------------------------------------------------------------------------
# instances that other sizes do not take
# --------------------------------------------------------------------------

@pytest.mark.parametrize("layout", ["nk", "kn"])
@pytest.mark.parametrize("K", [136, 1_024])
def test_floats_of_many_rows_in_small_tiles(K, layout):
    sizes = [512, 300, 0, 700, 1_100, 5, 900, 579]
    p = plan(8, sum(sizes), K, 1_032, F32, layout)
    assert (p.way, p.rows) == (TILES, 64)
    check(sizes, K, 1_032, F32, layout, k=2)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("K", [8, 136, 1_032])
def test_few_rows_of_two_tiles_of_columns(K, dtype):
    sizes = [1, 0, 3, 2, 8, 0, 20, 4]
    p = plan(8, sum(sizes), K, 2_056, dtype, "nk")
    assert (p.way, p.rows, p.columns) == (FEW, 16, 32)
    check(sizes, K, 2_056, dtype, "nk")
    check(sizes, K, 2_056, dtype, "nk", k=2, pad=8)


@pytest.mark.parametrize("dtype", TYPES)
def test_the_same_bits_on_every_call_by_tiles(dtype):
    sizes, K, N = [300, 0, 41, 1_700], 1_160, 2_056
    offsets, R = offsets_of(sizes).cuda(), sum(sizes)
    X, dY = random(1, R, K, dtype=dtype).cuda(), random(3, R, N, dtype=dtype).cuda()
    for layout in ("nk", "kn"):
        assert plan(4, R, K, N, dtype, layout).way == TILES and plan(4, R, K, N, dtype, layout, True).way == TILES
        W = weights(2, 4, K, N, dtype, layout).cuda()
        seen = None
        for _ in range(3):
            Y, dX, dW = torch.empty_like(dY), torch.empty_like(X), torch.empty_like(W)
            binding.sgap_grouped_mm(4, R, K, N, offsets, X, W, Y, layout)
            binding.sgap_grouped_mm(4, R, N, K, offsets, dY, W, dX, OTHER[layout])
            binding.sgap_grouped_mm_wgrad(4, R, K, N, offsets, X, dY, dW, layout)
            if seen is not None:
                assert all(torch.equal(a, b) for a, b in zip(seen, (Y, dX, dW)))
            seen = Y, dX, dW


# --------------------------------------------------------------------------
# floats in parts: the ends of their range
# --------------------------------------------------------------------------

R, N = 1_024, 1_600  # tiles enough for either layout


def product(X, W, layout, dtype=F32):
    K = X.shape[1]
    assert plan(1, R, K, N, dtype, layout).way == TILES
    Y = result(R, N, dtype)
    binding.sgap_grouped_mm(1, R, K, N, None, X.cuda(), W.cuda(), Y, layout)
    return Y


def gradient(X, dY, layout, dtype=F32):
    (rows, K), n = X.shape, dY.shape[1]
    assert plan(1, rows, K, n, dtype, layout, True).way == TILES
    dW = torch.full((1, n, K) if layout == "nk" else (1, K, n), float("nan"), dtype=dtype, device="cuda")
    binding.sgap_grouped_mm_wgrad(1, rows, K, n, None, X.cuda(), dY.cuda(), dW, layout)
    return dW


def check_product(X, W, layout, cut=0.0, dtype=F32):
    want, size = grouped_mm(offsets_of([R]), X, W, layout, R)
    assert_within(product(X, W, layout, dtype), want, torch.nan_to_num(size, 0, 0, 0) * (X.shape[1] + 4) * E + cut)


def check_gradient(X, dY, layout, dtype=F32):
    want, size = grouped_wgrad(offsets_of([len(X)]), X, dY, layout)
    assert_within(gradient(X, dY, layout, dtype), want, torch.nan_to_num(size, 0, 0, 0) * (len(X) + 4) * E)


LAYOUTS = pytest.mark.parametrize("layout", ["nk", "kn"])


@LAYOUTS
def test_floats_that_round_up_to_infinity_in_16_bits(layout):
    K = 72
    X, W = random(1, R, K), weights(2, 1, K, N, F32, layout, 2.0**-9)
    X[3, 5], X[70, 71], X[1_000, 64] = 3.4e38, -3.4028234e38, 3.4028234e38
    check_product(X, W, layout)
    X, W = random(3, R, K, scale=2.0**-9), weights(4, 1, K, N, F32, layout)
    W[0, 7, 9], W[0, -1, -1] = 3.4e38, -3.4e38
    check_product(X, W, layout)


@LAYOUTS
def test_gradients_of_floats_that_round_up_to_infinity_in_16_bits(layout):
    X, dY = random(1, 140, 1_160), random(2, 140, 1_152, scale=2.0**-9)
    X[3, 5], X[70, 71], X[139, 1_159] = 3.4e38, -3.4028234e38, 3.4028234e38
    check_gradient(X, dY, layout)


# a value that is no number, or infinite, makes those results so that it has a part in, and no others
@LAYOUTS
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("K", [64, 72, 200])
def test_values_that_are_no_numbers_by_tiles(K, dtype, layout):
    X, W = random(1, R, K, dtype=dtype), weights(2, 1, K, N, dtype, layout)
    X[3, K - 1], X[7, 0], X[130, 5], X[R - 1, K - 1] = float("inf"), float("nan"), float("-inf"), float("-inf")
    check_product(X, W, layout, dtype=dtype)
    column = W[0, 1_590] if layout == "nk" else W[0, :, 1_590]
    column[K - 1] = float("-inf")
    check_product(X, W, layout, dtype=dtype)


@LAYOUTS
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows", [128, 141])
def test_gradients_of_values_that_are_no_numbers_by_tiles(rows, dtype, layout):
    X, dY = random(1, rows, 1_160, dtype=dtype), random(2, rows, 1_152, dtype=dtype)
    X[rows - 1, 3], X[0, 1_159], dY[5, 700] = float("inf"), float("nan"), float("-inf")
    check_gradient(X, dY, layout, dtype)


# behind the last inner value and the last row the tiles hold zeros: values in memory there have no part in anything
@pytest.mark.parametrize("dtype", TYPES)
def test_what_lies_between_groups_and_rows_is_not_multiplied(dtype):
    sizes, K = [500, 0, 524], 72
    X, W = random(1, R, K, dtype=dtype), weights(2, 3, K, N, dtype, "nk")
    X[:500] = float("nan")
    W[1] = float("inf")
    assert plan(3, R, K, N, dtype, "nk").way == TILES
    Y = result(R, N, dtype)
    binding.sgap_grouped_mm(3, R, K, N, offsets_of(sizes).cuda(), X.cuda(), W.cuda(), Y, "nk")
    want, size = grouped_mm(offsets_of([524]), X[500:], W[2:], "nk", 524)
    assert torch.isnan(Y[:500]).all()
    assert_within(Y[500:], want, size * (K + 4) * E)
    X, dY = random(3, 280, 1_160, dtype=dtype), random(4, 280, 1_152, dtype=dtype)
    dY[:141] = float("inf")
    assert plan(2, 280, 1_160, 1_152, dtype, "nk", True).way == TILES
    dW = torch.full((2, 1_152, 1_160), float("nan"), dtype=dtype, device="cuda")
    binding.sgap_grouped_mm_wgrad(2, 280, 1_160, 1_152, offsets_of([141, 139]).cuda(), X.cuda(), dY.cuda(), dW, "nk")
    want, size = grouped_wgrad(offsets_of([139]), X[141:], dY[141:], "nk")
    assert_within(dW[1:], want, size * 143 * E)


@LAYOUTS
@pytest.mark.parametrize("scale", [1e-30, 1e-20, 1e15])
def test_floats_far_from_one(scale, layout):
    check_product(random(5, R, 72, scale=scale), weights(6, 1, 72, N, F32, layout, 1.0), layout)
    check_gradient(random(7, 140, 1_160, scale=scale), random(8, 140, 1_152), layout)


@LAYOUTS
def test_floats_under_the_range_of_16_bit_parts(layout):
    # below 2^-110 the last of the three parts is cut off at the smallest 16-bit number, 2^-133
    X, W = random(7, R, 72, scale=2.0**-112), weights(8, 1, 72, N, F32, layout, 1.0)
    cut = 2.0**-133 * W.double().abs().sum(2 if layout == "nk" else 1)
    check_product(X, W, layout, cut)


@LAYOUTS
def test_integers_of_24_bits_are_exact(layout):
    # one product to a sum: nothing is left out of a value
    K = 64
    X = torch.zeros(R, K)
    X[torch.arange(R), torch.arange(R) % K] = torch.randint(-2**24, 2**24, (R,), generator=torch.Generator().manual_seed(9)).float()
    W = torch.ones(1, *((N, K) if layout == "nk" else (K, N)))
    assert torch.equal(product(X, W, layout).cpu(), X.sum(1, keepdim=True).expand(R, N))


@LAYOUTS
def test_the_products_of_parts_that_are_left_out(layout):
    # 1 + 2^-8 - 2^-17 is 1, 2^-8 and -2^-17: what its square leaves out, middle x low twice and low x low, is 2^-24 of it.  Six
    # products of parts are added, each sum rounded by 2^-23 at most.
    K, value = 64, 1 + 2.0**-8 - 2.0**-17
    X, W = torch.zeros(R, K), torch.full((1, N, K) if layout == "nk" else (1, K, N), value)
    X[torch.arange(R), torch.arange(R) % K] = value
    got = product(X, W, layout).double().cpu()
    assert float((got - value**2).abs().max()) <= (1.1 * 2.0**-24 + 6 * 2.0**-23) * value**2
