"""Numbers of 8 bits with a scale for each block of 128: how values become codes, and products of them, against plain forms in
64 bits."""
import numpy as np
import pytest
import torch

from experts_util import E as EPS
from experts_util import assert_within, grouped_mm, offsets_of, random
from paper_2209_02882_amd import binding
from test_f8_plan import plan
from tokens_util import BLOCK, blocks, e4m3, f8_rows, f8_weights, filled, power_scale, random_codes, values

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.float16, torch.bfloat16]
F8 = torch.float8_e4m3fn


def to_rows(x):
    R, K = x.shape
    codes, scales = filled(F8, R, BLOCK * blocks(K)), filled(torch.float32, R, blocks(K))
    binding.sgap_f8_rows(R, K, x, codes, scales)
    return codes, scales


def to_weights(w, both=True):
    G, N, K = w.shape
    out = [filled(F8, G, N, BLOCK * blocks(K)), filled(torch.float32, G, blocks(N), blocks(K))]
    if both:
        out += [filled(F8, G, K, BLOCK * blocks(N)), filled(torch.float32, G, blocks(K), blocks(N))]
    binding.sgap_f8_weights(G, K, N, w, *out)
    return out


def same(codes, want):
    np.testing.assert_array_equal(codes.cpu().double().numpy(), want)


def extremes(dtype):
    """Blocks whose largest value is where the scale changes, of the type's smallest and largest numbers, ties, zeros, and some that
    are no finite numbers."""
    f = torch.finfo(dtype)
    x = torch.zeros(16, 300)
    x[0] = torch.linspace(-448, 448, 300)
    x[1, :10] = torch.tensor([448.0, 449.0, 464.0, 480.0, 447.0, 1.0625, 1.1875, 17.0, 19.0, -17.0])
    x[2] = 448.0 * 2.0**-5
    x[3] = (448.0 + 2.0) * 2.0**-6
    x[4] = f.max
    x[4, 1] = -f.max
    x[5] = f.tiny
    x[6] = f.smallest_normal * 3 / 4
    x[7, ::3] = f.max / 2
    x[7, 1::3] = f.tiny * 8
    x[8, 5], x[8, 140], x[8, 299] = float("nan"), float("inf"), -float("inf")
    x[8, 6], x[8, 150], x[8, 290] = 3.0, -5.0, 1e-3
    x[9] = float("nan")
    x[10, :128] = torch.arange(128) * 3.5          # 444.5 at most: ties between codes of 3 bits
    x[11, 128:256] = (torch.arange(128) - 64) * 2.0**-9 / 2   # codes without an exponent
    x[11, 128] = 448.0
    x[12, 0] = 1.75 * 2.0**8
    x[13, 0] = 1.7578125 * 2.0**8
    x[14, ::2] = -0.0
    x[15] = 2.0**-140 if dtype == torch.float32 else f.tiny
    return x.to(dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("R,K", [(1, 1), (3, 7), (2, 127), (5, 128), (4, 129), (17, 300), (33, 1001), (100, 2048), (1, 5000)])
def test_rows(R, K, dtype):
    x = (random(R + K, R, K) * torch.exp(2 * random(K, 1, K))).to(dtype)
    codes, scales = to_rows(x.cuda())
    want = f8_rows(x)
    np.testing.assert_array_equal(scales.cpu().double().numpy(), want[1])
    same(codes, want[0])


@pytest.mark.parametrize("dtype", TYPES)
def test_rows_of_extremes(dtype):
    x = extremes(dtype)
    codes, scales = to_rows(x.cuda())
    want = f8_rows(x)
    np.testing.assert_array_equal(scales.cpu().double().numpy(), want[1])
    same(codes, want[0])


@pytest.mark.parametrize("dtype", TYPES)
def test_rows_apart(dtype):
    x = random(1, 40, 333, dtype=dtype)
    held = x.cuda()
    for first in (0, 1, 2, 7):
        codes, scales = to_rows(held[:, first:first + 200])
        want = f8_rows(x[:, first:first + 200])
        np.testing.assert_array_equal(scales.cpu().double().numpy(), want[1])
        same(codes, want[0])


# every code: values at, half way between and a little beside neighbouring codes, in one block with 448
def test_every_rounding():
    code = torch.arange(127, dtype=torch.uint8).view(F8).double()
    middle = (code[1:] + code[:-1]) / 2
    x = torch.cat([torch.cat([v, -v]) for v in (code, middle, middle * (1 + 2.0**-20), middle * (1 - 2.0**-20))]).float()
    x = torch.nn.functional.pad(x, (0, -len(x) % 127)).view(-1, 127)
    x = torch.cat([x, torch.full((len(x), 1), 448.0)], dim=1)
    codes, scales = to_rows(x.cuda())
    assert (scales == 1).all()
    same(codes, e4m3(x.double().numpy()))
    assert torch.equal(codes.cpu().float(), x.to(F8).float())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("G,N,K", [(1, 1, 1), (2, 3, 130), (1, 128, 128), (3, 129, 127), (2, 200, 300), (1, 500, 64), (4, 70, 1001)])
@pytest.mark.parametrize("both", [False, True])
def test_weights(G, N, K, dtype, both):
    w = (random(G + N, G, N, K) * torch.exp(random(N, 1, N, 1))).to(dtype)
    got = to_weights(w.cuda(), both)
    codes, scales = f8_weights(w)
    np.testing.assert_array_equal(got[1].cpu().double().numpy(), scales)
    same(got[0], codes)
    if both:
        np.testing.assert_array_equal(got[3].cpu().double().numpy(), scales.swapaxes(1, 2))
        turned = np.zeros((G, K, blocks(N) * BLOCK))
        turned[:, :, :N] = codes[:, :, :K].swapaxes(1, 2)
        same(got[2], turned)


@pytest.mark.parametrize("dtype", TYPES)
def test_weights_of_extremes(dtype):
    w = extremes(dtype).view(1, 16, 300)
    got = to_weights(w.cuda())
    codes, scales = f8_weights(w)
    np.testing.assert_array_equal(got[1].cpu().double().numpy(), scales)
    same(got[0], codes)


# more weights than go through the caches: the same as of each matrix by itself, which is few enough
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N,K", [(4_700, 4_801), (4_699, 4_808)])
def test_weights_past_the_caches(N, K, dtype):
    assert 3 * N * K >= 1 << 26 > N * K
    w = torch.randn(3, N, K, generator=torch.Generator("cuda").manual_seed(K), device="cuda").to(dtype)
    for both in (True, False):
        all_of = to_weights(w, both)
        for g in range(3):
            for whole, alone in zip(all_of, to_weights(w[g:g + 1], both)):
                assert torch.equal(whole[g].view(torch.uint8), alone[0].view(torch.uint8))


def test_scales_are_the_smallest_powers():
    for most in (448.0, 448.00003, 447.99997, 1.0, 1e-38, 1e-45, 3.4e38, 0.0):
        s = power_scale(np.array([float(np.float32(most))]))[0]
        assert np.float32(most) <= 448 * s
        assert most == 0 or s == 2.0**-126 or np.float32(most) > 448 * (s / 2)
        x = torch.zeros(1, 128)
        x[0, 77] = -most
        assert to_rows(x.cuda())[1].item() == s


def operands(seed, x_rows, G, N, K):
    gen = torch.Generator().manual_seed(seed)
    x, w = random_codes(gen, x_rows, BLOCK * blocks(K), K=K), random_codes(gen, G, N, BLOCK * blocks(K), K=K)
    xs = torch.exp(torch.randn(x_rows, blocks(K), generator=gen)) / 448
    ws = torch.exp(torch.randn(G, blocks(N), blocks(K), generator=gen)) / 448   # (results fit float16)
    return x, xs, w, ws


def cut_off(dtype, bounds, x, xs, w, ws, K, R, src=None, src_div=1):
    """What results of 16 bits may lose beyond that: of eight neighbouring products seven times 2^-13 of the largest."""
    if dtype == torch.float32:
        return 0.0
    eights = lambda v: torch.nn.functional.pad(v.abs(), (0, -v.shape[-1] % 8)).unflatten(-1, (-1, 8)).amax(-1)  # noqa: E731
    return 7 * 2.0**-13 * grouped_mm(bounds, eights(values(x, xs, K, True)), eights(values(w, ws, K, False)), "nk", R, src, src_div)[1]


def product(x, xs, w, ws, K, offsets, R, dtype, src=None, src_div=1, columns=None):
    G, N = w.shape[:2]
    y = filled(dtype, R, N) if columns is None else columns
    binding.sgap_grouped_mm_f8(G, R, K, N, None if offsets is None else offsets.cuda(), x.cuda(), xs.cuda(), w.cuda(), ws.cuda(), y,
                               src=None if src is None else src.cuda(), src_div=src_div)
    return y


def check(x, xs, w, ws, K, offsets, R, dtype, src=None, src_div=1, what=""):
    got = product(x, xs, w, ws, K, offsets, R, dtype, src, src_div)
    bounds = offsets if offsets is not None else torch.tensor([0, R], dtype=torch.int32)
    want, size = grouped_mm(bounds, values(x, xs, K, True), values(w, ws, K, False), "nk", R, src, src_div)
    # products of codes are exact; K sums and two products of scales, in 32 bits
    assert_within(got, want, (K + 8) * EPS * size + cut_off(dtype, bounds, x, xs, w, ws, K, R, src, src_div), what)
    last = int(bounds[-1])
    if last < R:
        assert not torch.signbit(got[last:]).any() and not got[last:].any()


SHAPES = [  # sizes of groups, rows behind them, N, K
    ([1], 0, 1, 1), ([1], 0, 16, 128), ([5], 2, 17, 130), ([16], 0, 256, 64), ([17], 0, 100, 513), ([33], 3, 131, 1000), ([0, 3, 0, 40, 1], 4, 77, 300),
    ([2] * 9, 0, 130, 2048), ([64], 0, 64, 256), ([100], 5, 260, 384), ([128, 128], 0, 128, 128), ([129, 0, 300, 1, 70], 9, 200, 640),
    ([500], 0, 333, 129), ([700], 1, 512, 1024), ([255, 257, 64], 0, 520, 257), ([1] * 40, 0, 33, 200),
]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("sizes,more,N,K", SHAPES)
def test_products(sizes, more, N, K, dtype):
    R = sum(sizes) + more
    check(*operands(R + N, R, len(sizes), N, K), K, offsets_of(sizes), R, dtype)


# every kernel that a product may take, asked of the plan
@pytest.mark.parametrize("G,R,N,K,dtype,want", [
    (1, 11, 100, 500, torch.bfloat16, (0, 16, 16, 0)), (1, 40, 1000, 4000, torch.float16, (0, 16, 16, 0)),
    (7, 18, 1902, 3021, torch.bfloat16, (0, 16, 16, 2)), (5, 40, 3000, 2300, torch.float32, (0, 16, 16, 2)),
    (1, 64, 4000, 4000, torch.float16, (0, 32, 32, 0)), (3, 300, 900, 1300, torch.float32, (0, 32, 32, 0)),
    (3, 100, 4000, 300, torch.bfloat16, (1, 64, 128, 0)), (5, 4100, 4000, 1100, torch.float16, (1, 128, 128, 0)),
    (1, 4000, 8100, 530, torch.bfloat16, (1, 256, 256, 0)), (3, 6000, 4000, 1100, torch.float16, (1, 256, 256, 0)),
    (3, 2000, 3900, 500, torch.float32, (1, 64, 128, 0)), (2, 3000, 3900, 1500, torch.float32, (1, 128, 128, 0)),
    (1, 700, 1000, 1100, torch.bfloat16, (2, 64, 128, 0)), (3, 500, 2000, 1700, torch.float16, (2, 64, 128, 0)),
    (1, 300, 900, 1300, torch.float32, (2, 64, 128, 0)), (4, 400, 4000, 1500, torch.float16, (2, 128, 128, 0)),
    (1, 900, 3900, 2200, torch.bfloat16, (2, 128, 128, 0)), (1, 900, 3900, 2200, torch.float32, (2, 128, 128, 0)),
])
@pytest.mark.parametrize("gathered", [False, True])
def test_products_by_every_kernel(G, R, N, K, dtype, want, gathered):
    assert plan(G, R, K, N, dtype, given=G > 1, src=gathered, compute_units=torch.cuda.get_device_properties(0).multi_processor_count) == want
    gen = torch.Generator().manual_seed(R)
    sizes = torch.distributions.Multinomial(R - 3, torch.rand(G, generator=gen) + 0.2).sample().int() if G > 1 else torch.tensor([R])
    src = torch.randperm(R, generator=gen).int() if gathered else None
    x, xs, w, ws = (t.cuda() for t in operands(R, (R + 1) // 2 if gathered else R, G, N, K))
    off = offsets_of(sizes.tolist()) if G > 1 else None
    y = product(x, xs, w, ws, K, off, R, dtype, src, 2 if gathered else 1).double()
    # in 64 bits on the device: too many for the host
    rows = values(x, xs, K, True)
    rows = rows[torch.div(src.long().cuda(), 2, rounding_mode="floor")] if gathered else rows
    u = {torch.float32: 2.0**-24, torch.float16: 2.0**-11, torch.bfloat16: 2.0**-8}[dtype]
    for g, (a, b) in enumerate(zip([0] if off is None else off[:-1].tolist(), [R] if off is None else off[1:].tolist())):
        wv, v = values(w[g:g + 1], ws[g:g + 1], K, False)[0].t().contiguous(), rows[a:b].contiguous()
        want, size = v @ wv, v.abs() @ wv.abs()
        slack = (K + 8) * EPS * size
        if dtype != torch.float32:
            eights = lambda z: torch.nn.functional.pad(z.abs(), (0, -K % 8)).unflatten(-1, (-1, 8)).amax(-1)  # noqa: E731
            slack = slack + 7 * 2.0**-13 * (eights(v) @ eights(wv.t()).t().contiguous())
        assert ((y[a:b] - want).abs() <= slack + u * (want.abs() + slack) + 2.0**-24).all()
    last = R if off is None else int(off[-1])
    assert not y[last:].any()


def test_rows_gathered_from_more_than_4_gib():
    K, N, R, x_rows = 4224, 512, 40_000, (1 << 20) + 5
    assert plan(1, R, K, N, torch.bfloat16, given=False, src=True, x_rows=x_rows) == (1, 128, 128, 1)
    _, _, w, ws = operands(1, 1, 1, N, K)
    some, scales, _, _ = operands(2, 64, 1, 1, K)
    x = torch.zeros(x_rows, K, dtype=torch.uint8, device="cuda")
    xs = torch.ones(x_rows, K // BLOCK, device="cuda")
    at = torch.cat([torch.arange(20), torch.arange(x_rows - 44, x_rows)])
    x[at.cuda()], xs[at.cuda()] = some.view(torch.uint8).cuda(), scales.cuda()
    which = torch.randint(0, 64, (R,), generator=torch.Generator().manual_seed(3))
    y = filled(torch.bfloat16, R, N)
    binding.sgap_grouped_mm_f8(1, R, K, N, None, x.view(F8), xs, w.cuda(), ws.cuda(), y, src=at[which].int().cuda())
    want, size = grouped_mm(torch.tensor([0, 64]), values(some, scales, K, True), values(w, ws, K, False), "nk", 64)
    lost = cut_off(torch.bfloat16, torch.tensor([0, 64]), some, scales, w, ws, K, 64)
    assert_within(y, want[which], ((K + 8) * EPS * size + lost)[which])


@pytest.mark.parametrize("R", [1, 2, 15, 16, 17, 31, 48, 63, 64, 65, 127, 128, 129, 256, 300, 1000])
def test_products_of_one_group_without_offsets(R):
    check(*operands(R, R, 1, 144, 320), 320, None, R, torch.float32)


@pytest.mark.parametrize("sizes,N,K,k", [([3, 0, 9, 4], 50, 200, 2), ([200, 56, 0, 144], 140, 256, 4), ([600, 424], 300, 130, 1),
                                         ([300, 0, 210], 1000, 1100, 2), ([900], 2000, 1300, 1)])
def test_rows_gathered_by_a_list(sizes, N, K, k):
    R = sum(sizes)
    x_rows = R // k
    gen = torch.Generator().manual_seed(R)
    src = torch.randperm(R, generator=gen).int()
    check(*operands(R, x_rows, len(sizes), N, K), K, offsets_of(sizes), R, torch.bfloat16, src, k)
    # entries that name no row, and one row for many
    src = torch.where(torch.rand(R, generator=gen) < 0.3, torch.tensor(-1, dtype=torch.int32), src)
    src[::9] = x_rows * k
    src[1::9] = 2**31 - 1
    src[2::9] = 5 % (x_rows * k)
    check(*operands(R, x_rows, len(sizes), N, K), K, offsets_of(sizes), R, torch.float32, src, k)


@pytest.mark.parametrize("R", [20, 300])
def test_no_rows_to_gather_from_gives_zeros(R):
    _, _, w, ws = operands(1, 1, 1, 70, 200)
    got = product(torch.empty(0, 256, dtype=torch.uint8).view(F8), torch.empty(0, 2), w, ws, 200, None, R, torch.float32,
                  torch.zeros(R, dtype=torch.int32))
    assert torch.equal(got, torch.zeros_like(got))


@pytest.mark.parametrize("R", [20, 300])
def test_no_inner_values_give_zeros(R):
    got = product(torch.empty(R, 0, dtype=torch.uint8).view(F8), torch.empty(R, 0), torch.empty(1, 70, 0, dtype=torch.uint8).view(F8), torch.empty(1, 1, 0),
                  0, None, R, torch.float16)
    assert torch.equal(got, torch.zeros_like(got))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("R,N", [(9, 37), (9, 36), (200, 130), (200, 132)])
def test_results_apart(R, N, dtype):
    x, xs, w, ws = operands(3, R, 1, N, 384)
    want, size = grouped_mm(torch.tensor([0, R]), values(x, xs, 384, True), values(w, ws, 384, False), "nk", R)
    for first, pitch in [(0, N + 4), (1, N + 5), (3, N + 3), (4, N + 8)]:
        y = filled(dtype, R, pitch)
        product(x, xs, w, ws, 384, None, R, dtype, columns=y[:, first:first + N])
        lost = cut_off(dtype, torch.tensor([0, R]), x, xs, w, ws, 384, R)
        assert_within(y[:, first:first + N].contiguous(), want, 400 * EPS * size + lost)
        assert torch.isnan(y[:, :first]).all() and torch.isnan(y[:, first + N:]).all()


@pytest.mark.parametrize("R,N,K", [(12, 90, 256), (150, 90, 256), (300, 900, 1100)])
def test_nan_stays_in_its_row_and_column(R, N, K):
    if N == 900:  # teams, with an odd number of blocks
        assert plan(1, R, K, N, torch.float32, given=False)[0] == 2
    x, xs, w, ws = operands(2, R, 1, N, K)
    x.view(torch.uint8)[5, K - 56] = 0x7f
    w.view(torch.uint8)[0, 33, 7] = 0xff
    got = torch.isnan(product(x, xs, w, ws, K, None, R, torch.float32)).cpu()
    want = torch.zeros_like(got)
    want[5], want[:, 33] = True, True
    assert torch.equal(got, want)


@pytest.mark.parametrize("R", [3, 130, 400])
def test_sums_of_whole_numbers_are_exact(R):
    # codes -8 .. 8, scales of 1: every sum is a whole number below 2^24
    gen = torch.Generator().manual_seed(R)
    x, w = (torch.randint(-8, 9, s, generator=gen).float().to(F8) for s in ((R, 1024), (1, 96, 1024)))
    got = product(x, torch.ones(R, 8), w, torch.ones(1, 1, 8), 1024, None, R, torch.float32)
    assert torch.equal(got.cpu().double(), x.double() @ w[0].double().t())


@pytest.mark.parametrize("R", [8, 256])
def test_one_large_and_many_small_products_of_a_block(R):
    # 448 * 448 beside 127 products of 2^-6 * 2^-6 or less in a block: the sum holds them to 2^-23 of its size
    gen = torch.Generator().manual_seed(R)
    x, w = (torch.randint(1, 24, s, generator=gen).to(torch.uint8).view(F8) for s in ((R, 256), (1, 64, 256)))
    x.view(torch.uint8)[:, 3] = 0x7e
    w.view(torch.uint8)[:, :, 3] = 0x7e
    check(x, torch.ones(R, 2), w, torch.ones(1, 1, 2), 256, None, R, torch.float32)


@pytest.mark.parametrize("R", [2, 200])
def test_scales_of_extreme_size(R):
    x, _, w, _ = operands(1, R, 1, 40, 384)
    xs = torch.tensor([2.0**-126, 2.0**60, 1.0]).repeat(R, 1)
    ws = torch.tensor([[[2.0**100, 2.0**-100, 0.0]]])
    check(x, xs, w, ws, 384, None, R, torch.float32)
    ws = torch.tensor([[[-1.0, 3e-12, 1e-30]]])
    check(x, xs, w, ws, 384, None, R, torch.float32)


def test_a_training_step_of_experts():
    """Quantised, multiplied, and the gradient of the rows back, in the order in which a program calls them."""
    T, k, sizes, K, N = 150, 2, [120, 0, 80, 100], 200, 260
    R, G = T * k, len(sizes)
    offsets, src = offsets_of(sizes), torch.randperm(R, generator=torch.Generator().manual_seed(1)).int()
    x, w, dy = random(1, T, K, dtype=torch.bfloat16), random(2, G, N, K, scale=K**-0.5, dtype=torch.bfloat16), random(3, R, N, dtype=torch.bfloat16)
    xc, xs = to_rows(x.cuda())
    wc, ws, tc, ts = to_weights(w.cuda())
    dc, ds = to_rows(dy.cuda())
    y, dx = filled(torch.bfloat16, R, N), filled(torch.bfloat16, R, K)
    binding.sgap_grouped_mm_f8(G, R, K, N, offsets.cuda(), xc, xs, wc, ws, y, src=src.cuda(), src_div=k)
    binding.sgap_grouped_mm_f8(G, R, N, K, offsets.cuda(), dc, ds, tc, ts, dx)
    wv = torch.from_numpy(np.stack([f8_weights(w)[0][..., :K]])[0]) * torch.from_numpy(f8_weights(w)[1]).repeat_interleave(BLOCK, 1)[:, :N].repeat_interleave(BLOCK, 2)[..., :K]
    rows = lambda t, n: torch.from_numpy(f8_rows(t)[0][:, :n] * f8_rows(t)[1].repeat(BLOCK, axis=1)[:, :n])  # noqa: E731
    want, size = grouped_mm(offsets, rows(x, K), wv, "nk", R, src, k)
    assert_within(y, want, (K + 8) * EPS * size + cut_off(y.dtype, offsets, xc.cpu(), xs.cpu(), wc.cpu(), ws.cpu(), K, R, src, k))
    want, size = grouped_mm(offsets, rows(dy, N), wv, "kn", R)
    assert_within(dx, want, (N + 8) * EPS * size + cut_off(dx.dtype, offsets, dc.cpu(), ds.cpu(), tc.cpu(), ts.cpu(), N, R))


def test_captured_and_replayed():
    R, K, N = 300, 520, 200
    x, w = random(1, R, K).cuda(), random(2, 1, N, K).cuda()
    codes, scales, y = filled(F8, R, BLOCK * blocks(K)), filled(torch.float32, R, blocks(K)), filled(torch.float32, R, N)
    wc, ws = to_weights(w, both=False)

    def step():
        binding.sgap_f8_weights(1, K, N, w, wc, ws)
        binding.sgap_f8_rows(R, K, x, codes, scales)
        binding.sgap_grouped_mm_f8(1, R, K, N, None, codes, scales, wc, ws, y)

    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in (3, 4, 5):
        x.copy_(random(seed, R, K))
        w.copy_(random(seed + 10, 1, N, K))
        y.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        got = y.clone()
        step()
        assert torch.equal(got, y)
        c, s = f8_rows(x.cpu())
        wcode, wscale = f8_weights(w.cpu())
        want, size = grouped_mm(torch.tensor([0, R]), torch.from_numpy(c * s.repeat(BLOCK, axis=1))[:, :K],
                                torch.from_numpy(wcode * wscale.repeat(BLOCK, 1)[:, :N].repeat(BLOCK, 2))[..., :K], "nk", R)
        assert_within(got, want, (K + 8) * EPS * size)


def test_offsets_in_no_order_touch_nothing_else():
    R, N, K = 200, 70, 256
    x, xs, w, ws = operands(1, R, 3, N, K)
    for bad in ([0, 150, 40, 200], [-5, 1000, 30, 80], [2**31 - 1, -2**31, 0, 60]):
        y = filled(torch.float32, R + 2, N)
        product(x, xs, w, ws, K, torch.tensor(bad, dtype=torch.int32), R, torch.float32, columns=y[1:1 + R])
        assert torch.isnan(y[0]).all() and torch.isnan(y[-1]).all()


def test_other_types_and_lengths_are_refused():
    x, xs, w, ws = (t.cuda() for t in operands(1, 10, 1, 20, 200))
    y = torch.zeros(10, 20, device="cuda")
    with pytest.raises(TypeError, match="X must be"):
        binding.sgap_grouped_mm_f8(1, 10, 200, 20, None, x.view(torch.uint8), xs, w, ws, y)
    with pytest.raises(ValueError, match="w_scales"):
        binding.sgap_grouped_mm_f8(1, 10, 200, 20, None, x, xs, w, ws[..., :1].contiguous(), y)
    with pytest.raises(TypeError, match="Y must be"):
        binding.sgap_grouped_mm_f8(1, 10, 200, 20, None, x, xs, w, ws, y.double())
    with pytest.raises(ValueError, match="contiguous"):
        binding.sgap_f8_rows(10, 20, torch.zeros(20, 10, device="cuda").t(), x, xs)
    with pytest.raises(ValueError, match="codes"):
        binding.sgap_f8_rows(10, 20, y, x, xs[:, :1].contiguous())
    with pytest.raises(binding.SgapError, match="together"):
        binding.sgap_f8_weights(1, 200, 20, torch.zeros(1, 20, 200, device="cuda"), w, ws, codes_t=torch.zeros(1, 200, 128, dtype=torch.uint8, device="cuda").view(F8))
