"""Embeddings, the balance loss and numbers of 8 bits at the sizes from which on they take other kernels than small calls do, with
arrays beyond 2^31 elements, and with neighbours that nobody may touch."""
import numpy as np
import pytest
import torch

from experts_util import E as EPS
from experts_util import assert_within, grouped_mm, offsets_of, random
from paper_2209_02882_amd import binding
from test_f8_plan import plan
from test_gpu_balance import chosen, forward, gradient
from test_gpu_embed import draw_ids, workspace
from test_gpu_f8 import F8, TYPES, check, cut_off, extremes, operands, same, to_rows
from tokens_util import BLOCK, balance, blocks, embed, embed_grad, f8_rows, filled, values

pytestmark = pytest.mark.gpu


# ---- numbers of 8 bits: rows

# from 65,536 blocks on, where 8 divides a row's length, a thread has two blocks: that many, odd numbers of them, rows that end inside a
# block; one block less, which goes by one
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("R,K", [(65_536, 128), (65_535, 128), (8_193, 1_024), (6_001, 1_400), (65_539, 8), (13, 650_000)])
def test_rows_of_many_blocks(R, K, dtype):
    assert K % 8 == 0 and R * blocks(K) >= 65_535
    x = (random(R, R, K) * torch.exp(2 * random(K, 1, K))).to(dtype)
    edge = extremes(dtype)[:, :K][:R]
    x[-len(edge):, -edge.shape[1]:] = edge
    codes, scales = to_rows(x.cuda())
    want = f8_rows(x)
    np.testing.assert_array_equal(scales.cpu().double().numpy(), want[1])
    same(codes, want[0])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("first", [0, 1, 5])
def test_rows_of_many_blocks_apart(first, dtype):
    R, K = 11_003, 760
    assert R * blocks(K) >= 65_536
    x = random(3, R, K + 9, dtype=dtype)
    codes, scales = to_rows(x.cuda()[:, first:first + K])
    want = f8_rows(x[:, first:first + K])
    np.testing.assert_array_equal(scales.cpu().double().numpy(), want[1])
    same(codes, want[0])


# ---- embeddings

def whole(seed, *shape, dtype=torch.float32):
    """Whole numbers, whose sums floats hold in any order."""
    return torch.randint(-8, 9, shape, generator=torch.Generator().manual_seed(seed)).to(dtype)


# workgroups of groups of lanes that have a token each: from 2,048 on they have two
def lookup_workgroups(T, D, dtype):
    vec = 128 // torch.finfo(dtype).bits
    pieces = -(-D // vec) if D >= vec else D
    lanes = 1
    while lanes < 64 and lanes < pieces:
        lanes *= 2
    return -(-T * -(-pieces // lanes) * lanes // 256)


# odd numbers of tokens, whose last group has one; lengths that a piece of 16 bytes divides, does not, and is longer than
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("D", [2_048, 520, 513, 64, 5])
@pytest.mark.parametrize("apart,scale", [(0, 1.0), (5, -2.75)])
def test_lookup_of_two_tokens_to_a_group(D, apart, scale, dtype):
    T = 2_049
    while lookup_workgroups(T, D, dtype) < 2_048:
        T = 2 * T + 1
    V = 300
    ids, w = draw_ids("mixed", T, V), random(T + V, V, D, dtype=dtype)
    ids[-1], ids[-2], ids[0] = V - 1, -1, 0
    held = filled(dtype, T + 1, D + apart)
    out = held[:T, apart // 2:apart // 2 + D]
    binding.sgap_embed(T, V, D, ids.cuda(), w.cuda(), out, scale=scale)
    want = embed(ids, w, scale)
    assert_within(out.contiguous(), want, 2.0**-24 * want.abs())   # the scale's product in 32 bits
    assert not torch.signbit(out[((ids < 0) | (ids >= V)).cuda()]).any()
    assert torch.isnan(held[T]).all() and torch.isnan(held[:, :apart // 2]).all() and torch.isnan(held[:, apart // 2 + D:]).all()


# runs of more than eight tiles beyond their first, which a whole workgroup of the joins adds up, added to what is there; beside them runs
# of other lengths, rows without a token, rows whose last piece reaches back
@pytest.mark.parametrize("dtype,grad_dtype", [(torch.float32, torch.float32), (torch.float16, torch.float16), (torch.bfloat16, torch.bfloat16),
                                              (torch.float16, torch.float32), (torch.bfloat16, torch.float32)])
@pytest.mark.parametrize("T,V,D,runs", [(20_000, 9, 2_050, [19_000, 900]), (20_000, 9, 1_001, [12_000, 7_000, 1, 64]), (40_000, 5, 24, [39_000, 800]),
                                        (9_001, 1_003, 136, [8_500]), (30_000, 4, 3, [29_999])])
def test_long_runs_are_added(T, V, D, runs, dtype, grad_dtype):
    assert T > 8_192   # three launches
    ids = torch.full((T,), -1, dtype=torch.int32)
    at = torch.randperm(T, generator=torch.Generator().manual_seed(D))
    begin = 0
    for i, n in enumerate(runs):
        ids[at[begin:begin + n]] = (V - 1 - 2 * i) % V
        begin += n
    d, was = whole(1, T, D, dtype=dtype), whole(2, V, D, dtype=grad_dtype) / 4
    held = filled(grad_dtype, V + 2, D)
    grad = held[1:V + 1]
    grad.copy_(was)
    binding.sgap_embed_grad(T, V, D, ids.cuda(), d.cuda(), grad, scale=-0.375, accumulate=True, workspace=workspace(T, V, D))
    want, size, tokens = embed_grad(ids, d, V, -0.375)
    none = tokens[:, 0] == 0
    assert torch.equal(grad.cpu()[none], was[none])
    assert size.max() + was.abs().max() < 2**21   # multiples of an eighth: nothing is rounded but the result
    assert_within(grad, want + was.double(), 0.0)
    assert torch.isnan(held[0]).all() and torch.isnan(held[V + 1]).all()


# ids of one residue of the numbers of workgroups that the gradient of few tokens has
@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("T,V,step", [(5_003, 65_537, 256), (8_192, 65_536, 4_096), (700, 4_000_000, 4_096), (3_000, 50_001, 64)])
def test_gradient_of_ids_of_one_residue(T, V, step, accumulate):
    D = 40
    ids = (draw_ids("uniform", T, V) // step * step).clamp(max=V - 1)
    d, was = whole(1, T, D, dtype=torch.float16), whole(2, V, D) if accumulate else torch.zeros(V, D)
    grad = was.cuda() if accumulate else filled(torch.float32, V, D)
    binding.sgap_embed_grad(T, V, D, ids.cuda(), d.cuda(), grad, accumulate=accumulate, workspace=workspace(T, V, D))
    want, _, _ = embed_grad(ids, d, V, 1.0)
    assert torch.equal(grad.cpu().double(), want + was.double())


def test_tokens_rows_beyond_32_bits():
    # rows by token of 4.3 GB, forth and back; gradients are whole numbers, whose sums floats hold whatever their order
    T, V, D = (1 << 19) + 1, 50, 4_104
    gen = torch.Generator("cuda").manual_seed(1)
    ids = torch.randint(-1, V, (T,), generator=gen, device="cuda", dtype=torch.int32)
    ids[-1], ids[-2] = V - 1, 3
    w = torch.randint(-9, 10, (V, D), generator=gen, device="cuda").half()
    rows = torch.full((T, D), float("nan"), dtype=torch.float16, device="cuda")
    binding.sgap_embed(T, V, D, ids, w, rows)
    want, grad = torch.zeros(V, D, dtype=torch.float64, device="cuda"), filled(torch.float32, V, D)
    for a in range(0, T, 1 << 15):
        some = ids[a:a + (1 << 15)].long()
        part = torch.where((some >= 0)[:, None], w[some.clamp(min=0)], torch.zeros((), dtype=torch.float16, device="cuda"))
        assert torch.equal(rows[a:a + (1 << 15)], part)
        # (each token's row times one to three, so that tokens of one id differ)
        more = (torch.arange(a, a + len(some), device="cuda") % 3 + 1).half()[:, None]
        rows[a:a + (1 << 15)] = part * more
        want += torch.zeros(V + 1, D, dtype=torch.float64, device="cuda").index_add_(0, torch.where(some >= 0, some, V), (part * more).double())[:V]
    assert want.abs().max() < 2**24
    binding.sgap_embed_grad(T, V, D, ids, rows, grad, workspace=workspace(T, V, D))
    assert torch.equal(grad.double(), want)
    binding.sgap_embed_grad(T, V, D, ids, rows, grad, accumulate=True, workspace=workspace(T, V, D))
    assert torch.equal(grad.double(), 2 * want)


# ---- balance loss

def balance_parts(T, E, S, segments):
    """Workgroups to a sequence, as the rule has it."""
    tiles = -(-T // 64) + min(S, T) + 1
    part = 64 if tiles // S * E >= 65_536 else min(E, 256 if S >= 512 else 1_024)
    return -(-E // part)


# one sequence, or few, with so much to read that each 64 experts are a workgroup's: experts that 64 does not divide, one beyond it,
# 64 alone; sequences of very different lengths and an empty one
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("sizes,E,k", [([11_905], 353, 3), ([4_225], 1_000, 2), ([64_600], 65, 1), ([65_600], 64, 2), ([8_000, 0, 4_600], 1_024, 1),
                                       ([12_000, 1], 700, 4)])
def test_loss_by_parts_of_the_experts(sizes, E, k, dtype):
    T, segments = sum(sizes), None if len(sizes) == 1 else offsets_of(sizes)
    assert balance_parts(T, E, len(sizes), segments) == -(-E // 64)
    logits = (random(T, T, E, scale=1.5) + random(E, E)).to(dtype)
    experts = chosen(logits, k)
    on = None if segments is None else segments.cuda()
    loss, counts, rows = forward(logits.cuda(), experts.cuda(), on, k)
    want = balance(logits, experts, segments, k)
    np.testing.assert_array_equal(counts.cpu().numpy(), want[1])
    np.testing.assert_array_equal(rows.cpu().numpy(), want[2])
    # All terms are positive, so that a sum is off by its longest chain of additions: 16 values of a lane and 6 steps over lanes for a row's
    # exponentials, each off by its exponent's size and 4; 16 rows of a lane, 16 groups; T / 64 tiles by 16 lines, 16 lines; 22 for 64
    # experts, 16 parts, S sequences; products and quotients 8
    wide = float(logits.float().max() - logits.float().min())
    chain = 16 + 6 + wide + 4 + 16 + 16 + T / 64 / 16 + 16 + 22 + 16 + len(sizes) + 8
    assert_within(loss, np.array([want[0]]), chain * EPS * want[0], "loss")
    dlogits = gradient(logits.cuda(), experts.cuda(), on, k, counts, rows)
    assert_within(dlogits, want[3], (2 * 22 + 2 * wide + 32) * EPS * want[4], "gradient")


def test_more_logits_than_32_bits_count():
    # 64 tokens over and over: the loss is theirs, a token's gradient theirs by the number of turns
    E, k, turns = 1_024, 3, (1 << 15) + 1
    T = 64 * turns
    assert T * E > 1 << 31
    x = random(5, 64, E, dtype=torch.bfloat16)
    experts = chosen(x, k)
    logits, many = x.cuda().repeat(turns, 1), experts.cuda().repeat(turns, 1)
    loss, counts, rows = forward(logits, many, None, k)
    want = balance(x, experts, None, k)
    np.testing.assert_array_equal(counts.cpu().numpy(), want[1] * turns)
    assert rows.item() == T
    wide = float(x.float().max() - x.float().min())
    assert_within(loss, np.array([want[0]]), (160 + wide + T / 64 / 16) * EPS * want[0])
    dlogits = gradient(logits, many, None, k, counts, rows, dloss=float(turns))
    first = dlogits[:64].clone()
    assert_within(first, want[3], (2 * 22 + 2 * wide + 32) * EPS * want[4])
    for a in range(0, T, 1 << 16):
        part = dlogits[a:a + (1 << 16)].view(-1, 64, E)
        assert torch.equal(part, first.expand_as(part))


def guarded(dtype, *shape, before=64, behind=64):
    """(a contiguous tensor, check that nothing around it has been touched)"""
    n = int(np.prod(shape))
    value = 0x5a if dtype == torch.uint8 else -77 if dtype == torch.int32 else -2.5
    held = torch.full((before + n + behind,), value, dtype=dtype, device="cuda")

    def untouched():
        assert (held[:before] == value).all() and (held[before + n:] == value).all()

    return held[before:before + n].view(shape), untouched


# what such lists give is nothing that the header promises; all of it stays inside the arrays
@pytest.mark.parametrize("S", [3, 64, 70, 600, 4_100])
@pytest.mark.parametrize("E", [16, 130])
def test_segments_in_no_order_stay_inside_every_array(S, E):
    T, k = 500, 2
    rng = np.random.default_rng(S + E)
    x = random(1, T, E)
    experts = chosen(x, k).cuda()
    lists = [rng.integers(-50, T + 50, S + 1), rng.permutation(np.linspace(0, T, S + 1).astype(np.int64)), np.sort(rng.integers(0, T + 1, S + 1))[::-1],
             rng.choice([-2**31, 2**31 - 1, 0, T, T - 1, 7], S + 1)]
    for list_ in lists:
        segments = torch.from_numpy(np.ascontiguousarray(list_).astype(np.int32)).cuda()
        made = [guarded(torch.float32, 1), guarded(torch.int32, S, E), guarded(torch.int32, S),
                guarded(torch.uint8, binding.sgap_route_balance_workspace_size(T, E, k, S), before=256, behind=4_096), guarded(torch.float32, T, E, before=E, behind=E)]
        loss, counts, rows, ws, dlogits = (t for t, _ in made)
        binding.sgap_route_balance(T, E, k, S, x.cuda(), experts, segments, loss, counts, rows, workspace=ws)
        binding.sgap_route_balance_grad(T, E, k, S, x.cuda(), experts, segments, counts, rows, torch.ones(1, device="cuda"), dlogits)
        torch.cuda.synchronize()
        for _, untouched in made:
            untouched()
        assert (counts >= 0).all() and (rows >= 0).all()


# ---- products of numbers of 8 bits

# rows gathered from more than 4 GiB: every type of result; several groups, some empty, rows behind them; entries of two pairs a row, and
# some that name no row
@pytest.mark.parametrize("dtype", TYPES)
def test_groups_gathered_from_more_than_4_gib(dtype):
    K, N, sizes, x_rows, k = 4_224, 500, [14_000, 0, 21_111, 1, 4_800], (1 << 20) + 5, 2
    R, G = sum(sizes) + 9, len(sizes)
    assert plan(G, R, K, N, dtype, src=True, x_rows=x_rows) == (1, 128, 128, 1)
    some, scales, w, ws = operands(2, 64, G, N, K)
    x = torch.zeros(x_rows, K, dtype=torch.uint8, device="cuda")
    xs = torch.ones(x_rows, K // BLOCK, device="cuda")
    at = torch.cat([torch.arange(20), torch.arange(x_rows - 44, x_rows)])
    x[at.cuda()], xs[at.cuda()] = some.view(torch.uint8).cuda(), scales.cuda()
    gen = torch.Generator().manual_seed(3)
    which = torch.randint(0, 64, (R,), generator=gen)
    src = (at[which] * k + torch.randint(0, k, (R,), generator=gen)).int()
    src[::7], src[3::7] = -1, 2**31 - 1
    src[5::7] = x_rows * k   # the first that names none
    there = torch.ones(R, dtype=torch.bool)
    there[::7] = there[3::7] = there[5::7] = False
    offsets = offsets_of(sizes)
    y = filled(dtype, R, N)
    binding.sgap_grouped_mm_f8(G, R, K, N, offsets.cuda(), x.view(F8), xs, w.cuda(), ws.cuda(), y, src=src.cuda(), src_div=k)
    xv, wv = values(some, scales, K, True), values(w, ws, K, False)
    for g in range(G):
        a, b = int(offsets[g]), int(offsets[g + 1])
        want, size = grouped_mm(torch.tensor([0, 64]), xv, wv[g:g + 1], "nk", 64)
        lost = cut_off(dtype, torch.tensor([0, 64]), some, scales, w[g:g + 1], ws[g:g + 1], K, 64)
        real = there[a:b, None].double()
        assert_within(y[a:b], want[which[a:b]] * real, ((K + 8) * EPS * size + lost)[which[a:b]] * real, f"group {g}")
    assert not y[int(offsets[-1]):].any() and not torch.signbit(y[int(offsets[-1]):]).any() and not torch.signbit(y[(~there).cuda()]).any()


def test_rows_weights_and_results_beyond_32_bits():
    # Codes of 4.4 GB and results of 2.3 G elements: 64 rows over and over, so that results are theirs.  The last, odd, tile too.
    K, N, turns = 4_104, 2_100, (1 << 14) + 1
    R, pitch = 64 * turns + 3, blocks(K) * BLOCK
    assert R * pitch > 1 << 32 and R * N > 1 << 31
    x = random(1, 64, K, dtype=torch.bfloat16)
    held = torch.cat([x.cuda().repeat(turns, 1), x[:3].cuda()])
    codes, scales = to_rows(held)
    del held
    want_codes, want_scales = (torch.from_numpy(v) for v in f8_rows(x))
    for a in range(0, R - 3, 1 << 16):
        part = codes[a:min(a + (1 << 16), R - 3)].view(torch.uint8).view(-1, 64, pitch)
        assert torch.equal(part, part[:1].expand_as(part)) and torch.equal(part[0], codes[:64].view(torch.uint8))
    same(codes[:64], want_codes.numpy())
    same(codes[R - 3:], want_codes[:3].numpy())
    assert torch.equal(scales[:64].cpu().double(), want_scales) and torch.equal(scales[R - 3:].cpu().double(), want_scales[:3])
    _, _, w, ws = operands(4, 1, 1, N, K)
    assert plan(1, R, K, N, torch.bfloat16, given=False) == (1, 256, 256, 0)
    y = filled(torch.bfloat16, R, N)
    binding.sgap_grouped_mm_f8(1, R, K, N, None, codes, scales, w.cuda(), ws.cuda(), y)
    own, own_scales = codes[:64].cpu(), scales[:64].cpu()
    want, size = grouped_mm(torch.tensor([0, 64]), values(own, own_scales, K, True), values(w, ws, K, False), "nk", 64)
    slack = (K + 8) * EPS * size + cut_off(torch.bfloat16, torch.tensor([0, 64]), own, own_scales, w, ws, K, 64)
    assert_within(y[:64], want, slack)
    assert_within(y[R - 3:], want[:3], slack[:3])
    # (a row's sums go the same way in every tile)
    for a in range(0, R - 3, 1 << 16):
        part = y[a:min(a + (1 << 16), R - 3)].view(-1, 64, N)
        assert torch.equal(part, y[:64].expand_as(part))


@pytest.mark.parametrize("R", [24, 6_000])
def test_groups_of_weights_beyond_32_bits(R):
    # 4.4 GB of codes, as few rows and as tiles read them: rows of the last group and of the first
    G, N, K = 33, 16_400, 8_200
    pitch = blocks(K) * BLOCK
    assert G * N * pitch > 1 << 32
    x, xs, w, ws = operands(7, R, 1, N, K)
    codes = torch.zeros(G, N, pitch, dtype=torch.uint8, device="cuda")
    w_scales = torch.ones(G, blocks(N), blocks(K), device="cuda")
    codes[0], w_scales[0] = w[0].view(torch.uint8).cuda().flip(0), ws[0].cuda().flip(0)
    codes[G - 1], w_scales[G - 1] = w[0].view(torch.uint8).cuda(), ws[0].cuda()
    first = R // 3
    assert (plan(G, R, K, N, torch.bfloat16)[0] == 0) == (R == 24)
    offsets = torch.tensor([0] + [first] * (G - 1) + [R], dtype=torch.int32)
    y = filled(torch.bfloat16, R, N)
    binding.sgap_grouped_mm_f8(G, R, K, N, offsets.cuda(), x.cuda(), xs.cuda(), codes.view(F8), w_scales, y)
    xv = values(x, xs, K, True).cuda()
    some = torch.cat([torch.arange(0, 40), torch.arange(N - 40, N)])   # columns at both ends
    rows = torch.cat([torch.arange(0, min(12, first)), torch.arange(first, min(first + 12, R)), torch.arange(R - 5, R)])
    last = values(codes[G - 1].cpu().view(F8)[None], w_scales[G - 1].cpu()[None], K, False)[0][some]
    begin = values(codes[0].cpu().view(F8)[None], w_scales[0].cpu()[None], K, False)[0][some]
    eights = lambda v: torch.nn.functional.pad(v.abs(), (0, -v.shape[-1] % 8)).unflatten(-1, (-1, 8)).amax(-1)  # noqa: E731
    for r in rows.tolist():
        v, wv = xv[r].cpu(), begin if r < first else last
        size, lost = wv.abs() @ v.abs(), 7 * 2.0**-13 * (eights(wv) @ eights(v[None])[0])
        assert_within(y[r, some.cuda()], wv @ v, (K + 8) * EPS * size + lost, f"row {r}")


# results of 16 bits of few rows are made of exact products: what the tiles' instruction for codes may cut off is not left out of them
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("G,R,N,K", [(1, 11, 100, 500), (7, 18, 1_902, 3_021), (1, 64, 4_000, 4_000)])
def test_few_rows_are_exact(G, R, N, K, dtype):
    assert plan(G, R, K, N, dtype)[0] == 0
    sizes = [R // G] * (G - 1) + [R - R // G * (G - 1)]
    x, xs, w, ws = operands(R, R, G, N, K)
    offsets = offsets_of(sizes)
    y = filled(dtype, R, N)
    binding.sgap_grouped_mm_f8(G, R, K, N, offsets.cuda(), x.cuda(), xs.cuda(), w.cuda(), ws.cuda(), y)
    want, size = grouped_mm(offsets, values(x, xs, K, True), values(w, ws, K, False), "nk", R)
    assert_within(y, want, (K + 8) * EPS * size)
    check(x, xs, w, ws, K, offsets, R, torch.float32)


# every kernel of tiles, of 16-bit results, and few rows
KERNELS = [(11, 300, 500, (0, 16)), (60, 4_000, 4_000, (0, 32)), (700, 1_000, 1_100, (2, 64)), (900, 3_900, 2_200, (2, 128)), (300, 4_000, 300, (1, 64)),
           (2_000, 4_000, 4_000, (1, 128)), (4_000, 8_100, 530, (1, 256))]


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("R,N,K,kernel", KERNELS)
def test_products_that_nothing_cuts_off(R, N, K, kernel, dtype):
    # codes -8 .. 8: products lie within seven powers of two, which 13 bits hold whole, their sums are whole numbers below 2^24, and the
    # scales powers of two: a result is rounded once
    assert plan(1, R, K, N, dtype, given=False)[:2] == kernel
    gen = torch.Generator().manual_seed(R)
    pad = lambda v: torch.nn.functional.pad(v, (0, -K % BLOCK)).to(F8)  # noqa: E731
    x, w = (pad(torch.randint(-8, 9, s, generator=gen).float()) for s in ((R, K), (1, N, K)))
    y = filled(dtype, R, N)
    binding.sgap_grouped_mm_f8(1, R, K, N, None, x.cuda(), torch.full((R, blocks(K)), 0.25, device="cuda"), w.cuda(),
                               torch.full((1, blocks(N), blocks(K)), 0.5, device="cuda"), y)
    want = torch.mm(x.cuda().double(), w[0].cuda().double().t().contiguous()) / 8
    assert torch.equal(y, want.to(dtype))


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("R,N,K,kernel", KERNELS)
def test_nan_of_codes_stays_in_its_row_and_column(R, N, K, kernel, dtype):
    # a row that is NaN, a column with one in its last block, and rows that a list leaves out, in whose place the NaN row is read
    assert plan(1, R, K, N, dtype, given=False, src=True)[:2] == kernel
    x, xs, w, ws = operands(2, R, 1, N, K)
    x.view(torch.uint8)[0, :K] = 0x7f
    x.view(torch.uint8)[7, K - 1] = 0xff
    w.view(torch.uint8)[0, N - 2, K - 1] = 0x7f
    src = torch.arange(R, dtype=torch.int32)
    src[3], src[R - 2] = -1, R
    y = filled(dtype, R, N)
    y.zero_()
    binding.sgap_grouped_mm_f8(1, R, K, N, None, x.cuda(), xs.cuda(), w.cuda(), ws.cuda(), y, src=src.cuda())
    want = torch.zeros(R, N, dtype=torch.bool)
    want[0], want[7], want[:, N - 2] = True, True, True
    want[3], want[R - 2] = False, False
    assert torch.equal(torch.isnan(y).cpu(), want)
    assert not y[3].any() and not y[R - 2].any()
