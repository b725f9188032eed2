"""Sizes that make the products over groups take each of their tiles, and floats at the ends of their range."""
import numpy as np
import pytest
import torch

from experts_util import E, assert_within, grouped_mm, grouped_wgrad, offsets_of, random
from paper_2209_02882_amd import binding
from test_gpu_experts_products import check, check_w4, laid_out, result, w4_inputs

pytestmark = pytest.mark.gpu

HALVES = [torch.float16, torch.bfloat16]


# enough rows and columns for 256 x 256 (16-bit types) and 128 x 128 (floats); the rows' gradient has 72 or 200 columns
@pytest.mark.parametrize("layout", ["nk", "kn"])
@pytest.mark.parametrize("dtype", [torch.float32, *HALVES])
@pytest.mark.parametrize("K", [72, 200])
def test_many_rows_of_many_columns(K, dtype, layout):
    check([2000, 3111, 0, 1, 2500, 700], K, 4096, dtype, layout, extra=5)


# few rows of many weights: the gradient of the weights by 256 x 256
@pytest.mark.parametrize("layout", ["nk", "kn"])
@pytest.mark.parametrize("dtype", [torch.float32, *HALVES])
def test_many_weights(dtype, layout):
    check([65, 3, 0, 130, 64, 1, 7, 200, 0, 31, 33, 2], 1048, 1032, dtype, layout, k=2, extra=1)


# groups of half a large tile: 128 x 128 for 16-bit types
@pytest.mark.parametrize("dtype", HALVES)
def test_many_groups_of_128_rows(dtype):
    sizes = np.random.default_rng(5).integers(60, 196, 64).tolist()
    check(sizes, 64, 2048, dtype, "nk", k=1)


@pytest.mark.parametrize("dtype", HALVES)
@pytest.mark.parametrize("rows", [1, 2, 5, 17])
def test_w4_two_tiles_of_columns_to_a_wavefront(rows, dtype):
    sizes = [rows if g % 3 else 0 for g in range(64)]
    check_w4(sizes, 256, 205, 64, dtype, True, k=1)
    check_w4([rows], 128, 8200, 32, dtype, False, given=False)
    check_w4(sizes, 192, 205, 64, dtype, False, pad=1)


def run_f32(X, W, layout):
    R, K = X.shape
    N = W.shape[1] if layout == "nk" else W.shape[2]
    Y = result(R, N, torch.float32)
    binding.sgap_grouped_mm(1, R, K, N, None, X.cuda(), W.cuda(), Y, layout)
    return Y


@pytest.mark.parametrize("layout", ["nk", "kn"])
def test_floats_that_round_up_to_infinity_in_16_bits(layout):
    K, N, R = 64, 96, 140
    X, W = random(1, R, K), random(2, 1, *((N, K) if layout == "nk" else (K, N)), scale=2.0**-9)
    X[3, 5], X[70, 63] = 3.4e38, -3.4028234e38
    want, size = grouped_mm(offsets_of([R]), X, W, layout, R)
    assert_within(run_f32(X, W, layout), want, size * (K + 4) * E)
    # and the same value among the weights
    X, W = random(3, R, K, scale=2.0**-9), random(4, 1, *((N, K) if layout == "nk" else (K, N)))
    W[0, 7, 9] = 3.4e38
    want, size = grouped_mm(offsets_of([R]), X, W, layout, R)
    assert_within(run_f32(X, W, layout), want, size * (K + 4) * E)


@pytest.mark.parametrize("scale", [1e-30, 1e-20, 1e15])
def test_floats_far_from_one(scale):
    X, W = random(5, 130, 72, scale=scale), random(6, 1, 80, 72)
    want, size = grouped_mm(offsets_of([130]), X, W, "nk", 130)
    assert_within(run_f32(X, W, "nk"), want, size * 76 * E)


def test_floats_under_the_range_of_16_bit_parts():
    # below 2^-110 the last of the three parts is cut off at the smallest 16-bit number, 2^-133
    X, W = random(7, 130, 72, scale=2.0**-112), random(8, 1, 80, 72)
    want, size = grouped_mm(offsets_of([130]), X, W, "nk", 130)
    cut = 2.0**-133 * W.double().abs().sum(2)
    assert_within(run_f32(X, W, "nk"), want, size * 76 * E + cut)


def test_integers_of_24_bits_are_exact():
    # one product to a sum: nothing is left out of a value
    gen = torch.Generator().manual_seed(9)
    X = torch.zeros(128, 64)
    X[torch.arange(128), torch.arange(128) % 64] = torch.randint(-2**24, 2**24, (128,), generator=gen).float()
    W = torch.ones(1, 64, 64)
    assert torch.equal(run_f32(X, W, "nk").cpu(), X.sum(1, keepdim=True).expand(128, 64))


def test_the_same_bits_on_every_call():
    sizes, K, N = [300, 0, 41, 700], 264, 520
    offsets, R = offsets_of(sizes).cuda(), 1041
    for dtype in (torch.float32, *HALVES):
        X, W, dY = random(1, R, K, dtype=dtype).cuda(), random(2, 4, N, K, dtype=dtype).cuda(), random(3, R, N, dtype=dtype).cuda()
        seen = None
        for _ in range(3):
            Y, dW = torch.empty_like(dY), torch.empty_like(W)
            binding.sgap_grouped_mm(4, R, K, N, offsets, X, W, Y, "nk")
            binding.sgap_grouped_mm_wgrad(4, R, K, N, offsets, X, dY, dW, "nk")
            if seen is not None:
                assert torch.equal(seen[0], Y) and torch.equal(seen[1], dW)
            seen = Y, dW


@pytest.mark.parametrize("rows", [3, 30])
def test_w4_sums_that_are_infinite_by_definition(rows):
    K, N, group_k = 128, 16, 128
    codes, scales, _ = w4_inputs(1, K, N, group_k, torch.bfloat16, False)
    scales[:] = 1.0
    X = torch.zeros(rows, K, dtype=torch.bfloat16)
    X[1] = 3.0e38
    Y = result(rows, N, torch.bfloat16)
    binding.sgap_grouped_mm_w4(1, rows, K, N, group_k, None, X.cuda(), laid_out(1, K, N, group_k, codes, scales, None), Y)
    got = Y.float().cpu()
    assert (got[[r for r in range(rows) if r != 1]] == 0).all()
    # in the order of the inner dimension the running sum passes the largest float, and stays there or is no number
    assert not torch.isfinite(got[1]).any()


# few rows of few columns: the inner dimension shared by wavefronts, with blocks that are not whole
@pytest.mark.parametrize("dtype", [torch.float32, *HALVES])
@pytest.mark.parametrize("K", [8, 16, 24, 32, 120, 128, 136, 1024, 2056])
def test_few_rows_by_aligned_weights(K, dtype):
    for rows in (1, 2, 15, 16):
        check([rows], K, 88, dtype, "nk", given=False)
    check([3, 0, 1, 12, 8, 0, 0], K, 40, dtype, "nk", k=2, extra=3, pad=8)
    check([0, 2, 0], K, 2056, dtype, "nk", extra=1)


def test_few_rows_that_are_not_finite_stay_by_themselves():
    for K in (64, 72):
        X, W = torch.ones(6, K, dtype=torch.bfloat16), torch.ones(1, 24, K, dtype=torch.bfloat16)
        X[1, K - 1], X[4, 0] = float("inf"), float("nan")
        Y = result(6, 24, torch.bfloat16)
        binding.sgap_grouped_mm(1, 6, K, 24, None, X.cuda(), W.cuda(), Y, "nk")
        got = Y.float().cpu()
        assert (got[1] == float("inf")).all() and torch.isnan(got[4]).all() and (got[[0, 2, 3, 5]] == K).all()


# more rows, but too few tiles for the chip: two times sixteen rows to a wavefront
@pytest.mark.parametrize("dtype", [torch.float32, *HALVES])
@pytest.mark.parametrize("K,N", [(264, 104), (1024, 520)])
def test_few_tiles_by_aligned_weights(K, N, dtype):
    for rows in (17, 32, 33, 200):
        check([rows], K, N, dtype, "nk", given=False)
    check([40, 0, 33, 1], K, N, dtype, "nk", k=2, extra=40, pad=8)


# the same where a row of W is an inner value: a lane's pieces are put together from several rows
@pytest.mark.parametrize("dtype", [torch.float32, *HALVES])
@pytest.mark.parametrize("K", [8, 16, 24, 32, 120, 128, 136, 1024, 2056])
def test_few_rows_by_aligned_weights_of_the_other_layout(K, dtype):
    for rows in (1, 2, 15, 16, 17, 32, 33, 200):
        check([rows], K, 88, dtype, "kn", given=False)
    check([3, 0, 1, 12, 8, 0, 0], K, 40, dtype, "kn", k=2, extra=3, pad=8)
    check([40, 0, 33, 1], K, 104, dtype, "kn", k=2, extra=40, pad=8)
    check([0, 2, 0], K, 2056, dtype, "kn", extra=1)


def test_few_rows_that_are_not_finite_stay_by_themselves_in_the_other_layout():
    for K in (64, 72):
        X, W = torch.ones(6, K, dtype=torch.bfloat16), torch.ones(1, K, 24, dtype=torch.bfloat16)
        X[1, K - 1], X[4, 0], W[0, K - 1, 5] = float("inf"), float("nan"), float("-inf")
        Y = result(6, 24, torch.bfloat16)
        binding.sgap_grouped_mm(1, 6, K, 24, None, X.cuda(), W.cuda(), Y, "kn")
        got = Y.float().cpu()
        others = [c for c in range(24) if c != 5]
        assert torch.isnan(got[4]).all() and (got[[0, 1, 2, 3, 5], 5] == float("-inf")).all()
        assert (got[1, others] == float("inf")).all() and (got[[0, 2, 3, 5]][:, others] == K).all()


# more workgroups than compute units, where each has more columns
@pytest.mark.parametrize("layout", ["nk", "kn"])
@pytest.mark.parametrize("dtype", [torch.float32, *HALVES])
@pytest.mark.parametrize("K", [8, 136, 264])
def test_few_tiles_but_more_workgroups_than_compute_units(K, dtype, layout):
    check([600], K, 520, dtype, layout, given=False)
    check([2, 0, 5, 1, 8, 3, 1], K, 2056, dtype, layout, k=2, extra=3, pad=8)
    check([70, 0, 200, 1, 33], K, 1032, dtype, layout, extra=40)


# the gradient of few weights: rows shared by wavefronts, 64 x 64 weights to a workgroup
@pytest.mark.parametrize("layout", ["nk", "kn"])
@pytest.mark.parametrize("dtype", [torch.float32, *HALVES])
def test_gradient_of_few_weights(dtype, layout):
    check([300, 0, 71, 1], 520, 264, dtype, layout, k=2, extra=5)
    check([15, 16, 17, 0, 33], 264, 392, dtype, layout, pad=8)
    check([2100], 1160, 1032, dtype, layout, given=False)


# many groups of few rows, and columns enough for tiles of 64 x 128
@pytest.mark.parametrize("layout", ["nk", "kn"])
@pytest.mark.parametrize("dtype", [torch.float32, *HALVES])
@pytest.mark.parametrize("K", [8, 136])
def test_many_groups_of_few_rows_of_many_columns(K, dtype, layout):
    check([(7 * g) % 6 for g in range(40)], K, 2056, dtype, layout, k=2, extra=3, pad=8)


# rows of X that do not exist count as zeros in every kernel: few tiles (88 columns) and many
@pytest.mark.parametrize("layout", ["nk", "kn"])
@pytest.mark.parametrize("dtype", [torch.float32, *HALVES])
@pytest.mark.parametrize("N", [88, 89, 2056])
def test_missing_rows_of_x(N, dtype, layout):
    sizes, K, x_rows = [70, 0, 33, 200], 136, 60
    G, R, offsets = len(sizes), sum(sizes), offsets_of(sizes)
    src = torch.randint(-3, 2 * x_rows + 7, (R,), generator=torch.Generator().manual_seed(3)).int()
    src[5], src[6] = 2**31 - 1, -2**31
    X, dY = random(1, x_rows, K, dtype=dtype), random(3, R, N, dtype=dtype)
    W = random(2, *((G, N, K) if layout == "nk" else (G, K, N)), dtype=dtype, scale=K**-0.5)
    gone = (src < 0) | (src // 2 >= x_rows)
    # the plain form: an additional row of zeros for those that do not exist
    X0, src0 = torch.cat([X, torch.zeros(1, K, dtype=dtype)]), torch.where(gone, 2 * x_rows, src).int()
    Y, dW = result(R, N, dtype), torch.full_like(W, float("nan")).cuda()
    binding.sgap_grouped_mm(G, R, K, N, offsets.cuda(), X.cuda(), W.cuda(), Y, layout, src=src.cuda(), src_div=2)
    want, size = grouped_mm(offsets, X0, W, layout, R, src0, 2)
    assert_within(Y, want, size * (K + 4) * E)
    binding.sgap_grouped_mm_wgrad(G, R, K, N, offsets.cuda(), X.cuda(), dY.cuda(), dW, layout, src=src.cuda(), src_div=2)
    want, size = grouped_wgrad(offsets, X0, dY, layout, src0, 2)
    assert_within(dW, want, size * (max(sizes) + 4) * E)
