"""Products over ragged groups, their gradients, and the same with 4-bit weights, against plain 64-bit forms."""
import numpy as np
import pytest
import torch

from experts_util import (E, assert_within, grouped_mm, grouped_wgrad, offsets_of, random, w4_bound, w4_weights)
from paper_2209_02882_amd import binding

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.float16, torch.bfloat16]
OTHER = {"nk": "kn", "kn": "nk"}


def apart(t, pad, shift=0):
    """The same matrix on the device with rows `pad` elements further apart, `shift` elements from an aligned address; what
    lies between the rows is NaN."""
    rows, columns = t.shape
    flat = torch.full((rows * (columns + pad) + shift + 1,), float("nan"), dtype=t.dtype, device="cuda")
    view = flat[shift:shift + rows * (columns + pad)].view(rows, columns + pad)[:, :columns]
    view.copy_(t)
    return view


def result(R, N, dtype, pad=0, shift=0):
    return apart(torch.full((R, N), float("nan"), dtype=dtype), pad, shift)


def check(sizes, K, N, dtype, layout, k=0, extra=0, pad=0, shift=0, seed=1, given=True):
    """Forward and both gradients.  `extra`: rows behind the groups; `k`: rows are gathered, k of them from each row of X."""
    G, R = len(sizes), int(np.sum(sizes)) + extra
    offsets = offsets_of(sizes) if given else None
    src, div, x_rows = None, 1, R
    if k:
        x_rows = max(1, -(-R // k))
        gen = torch.Generator().manual_seed(seed)
        src, div = torch.randperm(x_rows * k, generator=gen)[:R].int(), k
    X = random(seed, x_rows, K, dtype=dtype)
    W = random(seed + 1, *((G, N, K) if layout == "nk" else (G, K, N)), dtype=dtype, scale=max(K, 1)**-0.5)
    dY = random(seed + 2, R, N, dtype=dtype)
    what = f"sizes {sizes[:8]} K {K} N {N} {dtype} {layout} k {k} pad {pad}"
    off_d, src_d = (None if t is None else t.cuda() for t in (offsets, src))
    gather = {} if src is None else dict(src=src_d, src_div=div)
    Xd, Wd, dYd = apart(X, pad, shift), W.cuda(), apart(dY, pad, shift)
    full = offsets if given else offsets_of([R])
    Y = result(R, N, dtype, pad, shift)
    binding.sgap_grouped_mm(G, R, K, N, off_d, Xd, Wd, Y, layout, **gather)
    want, size = grouped_mm(full, X, W, layout, R, src, div)
    assert_within(Y, want, size * (K + 4) * E, what + " Y")
    dX = result(R, K, dtype, pad, shift)
    binding.sgap_grouped_mm(G, R, N, K, off_d, dYd, Wd, dX, OTHER[layout])
    want, size = grouped_mm(full, dY, W, OTHER[layout], R)
    assert_within(dX, want, size * (N + 4) * E, what + " dX")
    dW = torch.full_like(Wd, float("nan"))
    binding.sgap_grouped_mm_wgrad(G, R, K, N, off_d, Xd, dYd, dW, layout, **gather)
    want, size = grouped_wgrad(full, X, dY, layout, src, div)
    longest = max(sizes) if len(sizes) else 0
    assert_within(dW, want, size * (longest + 4) * E, what + " dW")
    if pad:  # what lies between the rows is not written
        between = Y.as_strided((R, pad), (Y.stride(0), 1), Y.storage_offset() + N)
        assert torch.isnan(between).all()


SIZES = {
    "one row": [1], "a few": [3, 0, 2, 1], "around a tile": [31, 32, 33, 0, 127, 128, 129], "empty ends": [0, 0, 40, 0, 5, 0],
    "skewed": [700, 1, 0, 3, 0, 65], "all empty": [0, 0, 0],
}


@pytest.mark.parametrize("layout", ["nk", "kn"])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("sizes", list(SIZES))
@pytest.mark.parametrize("K,N", [(64, 128), (128, 96), (1, 1), (33, 65), (200, 40), (130, 257)])
def test_groups_and_sizes(sizes, K, N, dtype, layout):
    check(SIZES[sizes], K, N, dtype, layout)


@pytest.mark.parametrize("layout", ["nk", "kn"])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("K,N,pad,shift", [(64, 64, 8, 0), (72, 136, 0, 0), (64, 64, 1, 1), (100, 300, 3, 0), (8, 8, 0, 3), (256, 192, 16, 8)])
def test_gathered_rows_strides_and_rows_behind(K, N, pad, shift, dtype, layout):
    check([50, 0, 17, 140], K, N, dtype, layout, k=2, extra=9, pad=pad, shift=shift)
    check([5, 6], K, N, dtype, layout, k=3, extra=300, pad=pad, shift=shift)


@pytest.mark.parametrize("layout", ["nk", "kn"])
@pytest.mark.parametrize("dtype", TYPES)
def test_one_group_without_offsets(dtype, layout):
    for R in (1, 2, 15, 16, 17, 300):
        check([R], 160, 72, dtype, layout, given=False)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("layout", ["nk", "kn"])
@pytest.mark.parametrize("K,N", [(512, 512), (576, 1032), (1000, 531)])
def test_large_tiles(K, N, dtype, layout):
    check([700, 300, 0, 1100], K, N, dtype, layout, k=4, extra=3)
    check([513, 255], K, N, dtype, layout)


@pytest.mark.parametrize("dtype", TYPES)
def test_many_groups(dtype):
    rng = np.random.default_rng(3)
    check(rng.integers(0, 6, 200).tolist(), 72, 48, dtype, "nk", k=1, extra=5)
    check(rng.integers(0, 40, 130).tolist(), 64, 64, dtype, "kn")
    sizes = np.zeros(70, dtype=int)
    sizes[[63, 64, 69]] = 33, 1, 200
    check(sizes.tolist(), 64, 64, dtype, "nk")


@pytest.mark.parametrize("layout", ["nk", "kn"])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("K", [64, 65])
def test_infinities_stay_in_their_rows(K, dtype, layout):
    X, W = torch.ones(40, K, dtype=dtype), torch.ones(2, *((32, K) if layout == "nk" else (K, 32)), dtype=dtype)
    X[3, K - 1], X[7, 0] = float("inf"), float("nan")
    offsets = offsets_of([20, 20])
    Y = result(40, 32, dtype)
    binding.sgap_grouped_mm(2, 40, K, 32, offsets.cuda(), X.cuda(), W.cuda(), Y, layout)
    got = Y.float().cpu()
    assert (got[3] == float("inf")).all() and torch.isnan(got[7]).all()
    rest = [r for r in range(40) if r not in (3, 7)]
    assert (got[rest] == K).all()
    # the second group's gradient knows nothing of the first's rows
    dW = torch.full_like(W, 7).cuda()
    binding.sgap_grouped_mm_wgrad(2, 40, K, 32, offsets.cuda(), X.cuda(), torch.ones(40, 32, dtype=dtype).cuda(), dW, layout)
    assert (dW[1].float().cpu() == 20).all()


def test_rows_of_x_that_do_not_exist_count_as_zeros_and_offsets_may_overrun():
    X, W = torch.ones(6, 64, dtype=torch.bfloat16), torch.ones(2, 48, 64, dtype=torch.bfloat16)
    src = torch.tensor([0, 11, -1, 5, 12, 2**31 - 1, 3, 4], dtype=torch.int32)
    Y = result(8, 48, torch.bfloat16)
    binding.sgap_grouped_mm(2, 8, 64, 48, torch.tensor([0, 3, 50], dtype=torch.int32).cuda(), X.cuda(), W.cuda(), Y, "nk",
                            src=src.cuda(), src_div=2)
    assert Y[:, 0].float().tolist() == [64, 64, 0, 64, 0, 0, 64, 64]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_offsets_of_elements_beyond_32_bits(dtype):
    # rows 2^16 + 8 elements apart, the last ones more than 2^31 elements (4 GiB) from the first
    x_rows, K, N, ld = 36_000, 64, 72, (1 << 16) + 8
    flat = torch.empty(x_rows * ld, dtype=dtype, device="cuda")
    X = flat.view(x_rows, ld)[:, :K]
    X.normal_()
    src = torch.tensor([0, 1, x_rows - 1, x_rows - 2, 33_000, 32_768, 5] * 40, dtype=torch.int32)
    sizes = [100, 0, 180]
    W = random(3, 3, N, K, dtype=dtype, scale=0.1)
    rows = X[src.long().cuda()].cpu()
    Y = result(280, N, dtype)
    binding.sgap_grouped_mm(3, 280, K, N, offsets_of(sizes).cuda(), X, W.cuda(), Y, "nk", src=src.cuda())
    want, size = grouped_mm(offsets_of(sizes), rows, W, "nk", 280)
    assert_within(Y, want, size * (K + 4) * E)
    dY = random(4, 280, N, dtype=dtype)
    dW = torch.empty(3, N, K, dtype=dtype, device="cuda")
    binding.sgap_grouped_mm_wgrad(3, 280, K, N, offsets_of(sizes).cuda(), X, dY.cuda(), dW, "nk", src=src.cuda())
    want, size = grouped_wgrad(offsets_of(sizes), rows, dY, "nk")
    assert_within(dW, want, size * 190 * E)


def test_gradients_against_differences():
    # the product is linear in X and in W: a difference along a direction is the gradient's product with it, up to rounding
    sizes, K, N = [20, 0, 31], 48, 40
    offsets, R = offsets_of(sizes).cuda(), 51
    X, W, dY = random(1, R, K).cuda(), random(2, 3, N, K).cuda(), random(3, R, N).cuda()
    U, V = random(4, R, K).cuda(), random(5, 3, N, K).cuda()
    out = [torch.empty(R, N, device="cuda") for _ in range(4)]
    for y, x, w in zip(out, (X + U, X - U, X, X), (W, W, W + V, W - V)):
        binding.sgap_grouped_mm(3, R, K, N, offsets, x, w, y, "nk")
    dX, dW = torch.empty_like(X), torch.empty_like(W)
    binding.sgap_grouped_mm(3, R, N, K, offsets, dY, W, dX, "kn")
    binding.sgap_grouped_mm_wgrad(3, R, K, N, offsets, X, dY, dW, "nk")
    for (a, b), grad, along in (((out[0], out[1]), dX, U), ((out[2], out[3]), dW, V)):
        slope = ((a.double() - b.double()) / 2 * dY.double()).sum()
        exact = (grad.double() * along.double()).sum()
        size = (a.double().abs() * dY.double().abs()).sum() + (grad.double() * along.double()).abs().sum()
        assert abs(float(slope - exact)) <= 2 * 64 * E * float(size)


# --------------------------------------------------------------------------
# 4-bit weights
# --------------------------------------------------------------------------

def w4_inputs(G, K, N, group_k, dtype, zeros, seed=1):
    gen = torch.Generator().manual_seed(seed)
    codes = torch.randint(0, 256, (G, N, K // 2), generator=gen, dtype=torch.uint8)
    scales = (torch.rand(G, N, K // group_k, generator=gen) * 0.1 - 0.03).to(dtype)
    zero = torch.randint(0, 16, (G, N, K // group_k), generator=gen, dtype=torch.uint8) if zeros else None
    return codes, scales, zero


def laid_out(G, K, N, group_k, codes, scales, zero):
    size = binding.sgap_w4_layout_size(G, K, N, group_k, zeros=zero is not None)
    weights = torch.full((size,), 0xa5, dtype=torch.uint8, device="cuda")
    binding.sgap_w4_layout(G, K, N, group_k, codes.cuda(), scales.cuda(), None if zero is None else zero.cuda(), weights)
    return weights


def check_w4(sizes, K, N, group_k, dtype, zeros, k=0, extra=0, pad=0, shift=0, given=True, seed=1):
    G, R = len(sizes), int(np.sum(sizes)) + extra
    codes, scales, zero = w4_inputs(G, K, N, group_k, dtype, zeros, seed)
    weights = laid_out(G, K, N, group_k, codes, scales, zero)
    src, div, x_rows = None, 1, R
    if k:
        x_rows = max(1, -(-R // k))
        src, div = torch.randperm(x_rows * k, generator=torch.Generator().manual_seed(seed))[:R].int(), k
    X = random(seed + 5, x_rows, K, dtype=dtype)
    Y = result(R, N, dtype, pad, shift)
    offsets = offsets_of(sizes)
    binding.sgap_grouped_mm_w4(G, R, K, N, group_k, offsets.cuda() if given else None, apart(X, pad, shift), weights, Y, zeros=zeros,
                               **({} if src is None else dict(src=src.cuda(), src_div=div)))
    want, _ = grouped_mm(offsets, X, w4_weights(codes, scales, zero, group_k), "nk", R, src, div)
    _, size = grouped_mm(offsets, X, w4_bound(codes, scales, zero, group_k), "nk", R, src, div)
    assert_within(Y, want, size * (K + 8) * E, f"w4 {sizes[:8]} K {K} N {N} group {group_k} {dtype} zeros {zeros}")


@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("K,group_k", [(32, 32), (96, 32), (64, 64), (320, 64), (128, 128), (640, 128), (512, 256), (2048, 512)])
@pytest.mark.parametrize("N", [1, 16, 50])
def test_w4_scales_and_sizes(K, group_k, N, dtype, zeros):
    check_w4([1], K, N, group_k, dtype, zeros, given=False)
    check_w4([3, 0, 17, 1], K, N, group_k, dtype, zeros, k=2, extra=2)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("rows", [2, 8, 15, 16, 17, 33, 48, 49, 130])
def test_w4_rows(rows, dtype):
    check_w4([rows], 1024, 80, 64, dtype, True, given=False)
    check_w4([rows, 0, rows + 1], 256, 33, 128, dtype, False, pad=3, shift=1)


def test_w4_many_groups_and_long_rows():
    rng = np.random.default_rng(4)
    check_w4(rng.integers(0, 4, 150).tolist(), 256, 48, 64, torch.bfloat16, True, k=1)
    check_w4([900, 3], 128, 40, 32, torch.float16, False)
    check_w4([0, 0], 128, 40, 32, torch.float16, False, extra=4)
    check_w4([2], 8192, 24, 128, torch.bfloat16, True, given=False)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("rows", [4, 40])
def test_w4_rows_that_are_not_finite_or_overflow_on_the_way(rows, dtype):
    K, N, group_k = 256, 32, 64
    codes, scales, zero = w4_inputs(1, K, N, group_k, dtype, True)
    X = random(1, rows, K, dtype=dtype)
    X[1, 70] = float("inf")
    X[2, 3] = float("nan")
    if dtype == torch.bfloat16:
        X[3, 100] = 3.0e38  # 31 times that is no float, the weight's product is one
        scales[:, :, 1] = 2.0**-20
    Y = result(rows, N, dtype)
    binding.sgap_grouped_mm_w4(1, rows, K, N, group_k, None, X.cuda(), laid_out(1, K, N, group_k, codes, scales, zero), Y, zeros=True)
    W = w4_weights(codes, scales, zero, group_k)
    want, _ = grouped_mm(offsets_of([rows]), X, W, "nk", rows)
    _, size = grouped_mm(offsets_of([rows]), torch.nan_to_num(X, 0, 0, 0), w4_bound(codes, scales, zero, group_k), "nk", rows)
    assert_within(Y, want, size * (K + 8) * E)


# --------------------------------------------------------------------------
# streams and graphs
# --------------------------------------------------------------------------

def test_a_side_stream_and_a_graph_replayed():
    T, n, k, K, N = 200, 12, 3, 128, 96
    dtype = torch.bfloat16
    gen = torch.Generator().manual_seed(8)
    logits, X, W = torch.randn(T, n, generator=gen).cuda(), random(1, T, K, dtype=dtype).cuda(), random(2, n, N, K, dtype=dtype).cuda()
    codes, scales, _ = w4_inputs(n, K, N, 64, dtype, False)
    weights = laid_out(n, K, N, 64, codes, scales, None)
    i32 = dict(dtype=torch.int32, device="cuda")
    gates, experts, slot = torch.empty(T, k, device="cuda"), torch.empty(T, k, **i32), torch.empty(T, k, **i32)
    order, offsets = torch.empty(T * k, **i32), torch.empty(n + 1, **i32)
    workspace = torch.empty(binding.sgap_route_topk_workspace_size(T, n, k), dtype=torch.uint8, device="cuda")
    Y, Y4 = (torch.empty(T * k, N, dtype=dtype, device="cuda") for _ in range(2))
    out, dW, dgates = torch.empty(T, N, dtype=dtype, device="cuda"), torch.empty_like(W), torch.empty(T, k, device="cuda")
    dZ, dl = torch.empty_like(Y), torch.empty_like(logits)

    def work(stream=None):
        binding.sgap_route_topk(T, n, k, logits, gates, experts, slot, order, offsets, workspace=workspace, stream=stream)
        binding.sgap_grouped_mm(n, T * k, K, N, offsets, X, W, Y, "nk", src=order, src_div=k, stream=stream)
        binding.sgap_grouped_mm_w4(n, T * k, K, N, 64, offsets, X, weights, Y4, src=order, src_div=k, stream=stream)
        binding.sgap_route_combine(T, k, N, Y, slot, gates, out, stream=stream)
        binding.sgap_route_combine_grad(T, k, N, Y, slot, order, gates, out, dZ, dgates, stream=stream)
        binding.sgap_grouped_mm_wgrad(n, T * k, K, N, offsets, X, dZ, dW, "nk", src=order, src_div=k, stream=stream)
        binding.sgap_route_topk_grad(T, n, k, logits, gates, experts, dgates, dl, stream=stream)

    results = (gates, experts, slot, order, offsets, Y, Y4, out, dZ, dgates, dW, dl)

    def poison():
        for t in results:
            t.fill_(-3)

    def same(want):
        torch.cuda.synchronize()
        return all(torch.equal(a, b) for a, b in zip(results, want))

    work()
    torch.cuda.synchronize()
    first = [t.clone() for t in results]
    side = torch.cuda.Stream()
    poison()
    side.wait_stream(torch.cuda.current_stream())
    work(side)  # by argument
    torch.cuda.current_stream().wait_stream(side)
    assert same(first)
    poison()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        work()  # torch's current stream
    torch.cuda.current_stream().wait_stream(side)
    assert same(first)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        work()
    for seed in range(4):
        logits.copy_(torch.randn(T, n, generator=gen))
        X.copy_(random(seed, T, K, dtype=dtype))
        poison()
        graph.replay()
        torch.cuda.synchronize()
        replayed = [t.clone() for t in results]
        poison()
        work()
        assert same(replayed)
