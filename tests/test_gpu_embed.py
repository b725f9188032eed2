"""Rows of a table by token and the gradient of the table, against plain forms in 64 bits."""
import numpy as np
import pytest
import torch

from experts_util import E, U, assert_within, random
from paper_2209_02882_amd import binding
from tokens_util import embed, embed_grad, filled

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.float16, torch.bfloat16]


def draw_ids(kind, T, V, seed=0):
    rng = np.random.default_rng(seed)
    if kind == "uniform":
        ids = rng.integers(0, V, T)
    elif kind == "skewed":  # as words are: the first ones far more often than the others
        ids = np.minimum(np.exp(rng.uniform(0, np.log(V + 1), T)).astype(np.int64) - 1, V - 1)
    elif kind == "one":
        ids = np.full(T, V // 2)
    elif kind == "sorted":
        ids = np.sort(rng.integers(0, V, T))
    elif kind == "none":
        ids = np.where(np.arange(T) % 2, -1, V)
    else:  # some outside the table, at both ends and far away
        ids = np.where(rng.random(T) < 0.3, rng.choice([-1, V, -2**31, 2**31 - 1, V + 1], T), rng.integers(0, V, T))
    return torch.from_numpy(ids.astype(np.int32))


# The gradient of a few tokens goes in one launch, of more in three.  With so many tokens beside the real ones that no row has, and whose
# gradients are NaN, small sizes take the three.
OTHERS = [0, 8_300]


def among(others, ids, d):
    before, behind = torch.full((others // 3,), -1, dtype=torch.int32), torch.full((others - others // 3,), -1, dtype=torch.int32)
    nan = lambda n: torch.full((len(n), d.shape[1]), float("nan"), dtype=d.dtype)  # noqa: E731
    return (torch.cat([before, ids, behind]), torch.cat([nan(before), d, nan(behind)])) if others else (ids, d)


def workspace(T, V, D):
    return torch.full((binding.sgap_embed_grad_workspace_size(T, V, D),), 0x5a, dtype=torch.uint8, device="cuda")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,V,D,kind", [(1, 1, 1, "one"), (1, 50, 64, "uniform"), (7, 3, 5, "mixed"), (33, 1000, 8, "mixed"), (64, 10, 129, "skewed"),
                                        (100, 77, 1001, "mixed"), (513, 300, 512, "skewed"), (20, 5, 4100, "uniform"), (5, 9, 3, "none")])
@pytest.mark.parametrize("scale", [1.0, -2.75])
def test_rows_of_the_table(T, V, D, kind, dtype, scale):
    ids, w = draw_ids(kind, T, V), random(T + V, V, D, dtype=dtype)
    out = filled(dtype, T, D)
    binding.sgap_embed(T, V, D, ids.cuda(), w.cuda(), out, scale=scale)
    want = embed(ids, w, scale)
    assert_within(out, want, 2.0**-24 * want.abs())
    assert not torch.signbit(out[(ids < 0) | (ids >= V)]).any()


@pytest.mark.parametrize("dtype", TYPES)
def test_rows_apart_and_odd_addresses(dtype):
    T, V, D = 40, 30, 77
    ids, w = draw_ids("mixed", T, V), random(3, V, D + 13, dtype=dtype)
    held, out = w.cuda(), filled(dtype, T, D + 5)
    for first in (0, 1, 3):
        binding.sgap_embed(T, V, D, ids.cuda(), held[:, first:first + D], out[:, 2:2 + D])
        assert_within(out[:, 2:2 + D].contiguous(), embed(ids, w[:, first:first + D], 1.0), 0.0)
        assert torch.isnan(out[:, :2]).all() and torch.isnan(out[:, 2 + D:]).all()


def test_infinities_and_nan_of_a_row_stay_its_own():
    w = torch.tensor([[1.0, float("inf"), 2.0], [float("nan"), 3.0, -float("inf")], [4.0, 5.0, 6.0]])
    out = filled(torch.float32, 4, 3)
    binding.sgap_embed(4, 3, 3, torch.tensor([2, 0, -1, 1], dtype=torch.int32, device="cuda"), w.cuda(), out, scale=0.5)
    assert_within(out, torch.stack([w[2], w[0], torch.zeros(3), w[1]]).double() * 0.5, 0.0)


@pytest.mark.parametrize("others", OTHERS)
@pytest.mark.parametrize("dtype,grad_dtype", [(t, t) for t in TYPES] + [(torch.float16, torch.float32), (torch.bfloat16, torch.float32)])
@pytest.mark.parametrize("T,V,D,kind", [
    (1, 1, 1, "one"), (1, 700, 64, "uniform"), (31, 3, 5, "mixed"), (32, 4, 64, "one"), (33, 4, 64, "one"), (64, 2, 8, "sorted"), (65, 9, 129, "sorted"),
    (300, 40, 1001, "mixed"), (1000, 513, 96, "skewed"), (1025, 1500, 520, "skewed"), (2048, 1, 16, "one"), (700, 90, 8, "none"),
    (4096, 20000, 40, "skewed"), (3000, 5, 264, "uniform"), (129, 65, 4104, "skewed"),
])
def test_gradient(T, V, D, kind, dtype, grad_dtype, others):
    ids, d = among(others, draw_ids(kind, T, V, seed=T), random(T + V, T, D, dtype=dtype))
    grad, ws = filled(grad_dtype, V, D), workspace(len(ids), V, D)
    binding.sgap_embed_grad(len(ids), V, D, ids.cuda(), d.cuda(), grad, scale=0.75, workspace=ws)
    want, size, tokens = embed_grad(ids, d, V, 0.75)
    assert_within(grad, want, (tokens + 4) * E * size)
    assert not torch.signbit(grad[(tokens[:, 0] == 0).cuda()]).any()


# as few ids as there are rows for a wavefront, more, and as many as one launch deals with; tokens up to its limit and behind it; one
# id's that a whole workgroup adds up, all of them or beside others
@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("T,V,D,kind", [(4_097, 1_025, 24, "skewed"), (1_024, 262_150, 136, "skewed"), (1_025, 262_150, 136, "skewed"), (8_192, 300, 40, "skewed"), (8_193, 300, 40, "skewed"),
                                        (33, 3, 1_032, "one"), (3_000, 2, 2_056, "sorted"), (1_000, 300_007, 8, "skewed"), (50, 1 << 22, 8, "skewed"),
                                        (50, (1 << 22) + 1, 8, "skewed"), (700, 5_000, 520, "mixed"), (8_192, 70_001, 8, "uniform"), (64, 256, 5, "mixed")])
def test_gradient_of_few(T, V, D, kind, accumulate):
    ids, d = draw_ids(kind, T, V, seed=V), random(5, T, D, dtype=torch.bfloat16)
    was = random(2, V, D) if accumulate else torch.zeros(V, D)
    grad = was.cuda() if accumulate else filled(torch.float32, V, D)
    binding.sgap_embed_grad(T, V, D, ids.cuda(), d.cuda(), grad, scale=-0.5, accumulate=accumulate, workspace=workspace(T, V, D))
    want, size, tokens = embed_grad(ids, d, V, -0.5)
    assert_within(grad, want + was.double(), (tokens + 5) * E * (size + was.double().abs()))
    none = tokens[:, 0] == 0
    assert torch.equal(grad.cpu()[none], was[none]) and (accumulate or not torch.signbit(grad[none.cuda()]).any())


# more tokens than 1,024 tiles (of rows of 2,048, and fewer of longer ones) of 8 hold, so that tiles are longer; more ids than 256 ranges
# of 256; tokens of which one id's fill most tiles
@pytest.mark.parametrize("T,V,D,kind", [(9_000, 40, 2_056, "skewed"), (20_000, 9, 2_050, "one"), (40_000, 300, 24, "skewed"), (70_001, 3, 8, "uniform"),
                                        (200, 300_001, 16, "skewed"), (33_000, 70_000, 40, "skewed")])
def test_gradient_of_many(T, V, D, kind):
    ids, d = draw_ids(kind, T, V), random(5, T, D)
    grad, ws = filled(torch.float32, V, D), workspace(T, V, D)
    binding.sgap_embed_grad(T, V, D, ids.cuda(), d.cuda(), grad, workspace=ws)
    want, size, tokens = embed_grad(ids, d, V, 1.0)
    assert_within(grad, want, (tokens + 4) * E * size)


# long rows of which few are in use; side by side, which are cleared as one piece of memory, and apart; rows that no range divides
@pytest.mark.parametrize("apart", [0, 7])
@pytest.mark.parametrize("T,V,D,kind", [(8_193, 33_003, 513, "skewed"), (9_001, 36_005, 516, "mixed"), (1_100, 65_601, 520, "uniform")])
def test_gradient_of_few_rows_of_many(T, V, D, kind, apart):
    ids, d = draw_ids(kind, T, V), random(5, T, D, dtype=torch.bfloat16)
    ids[T // 2], ids[T // 3] = V - 1, -1
    held = filled(torch.float32, V + 2, D + apart)
    grad = held[1:V + 1, apart // 2:apart // 2 + D]
    binding.sgap_embed_grad(T, V, D, ids.cuda(), d.cuda(), grad, scale=-2.0, workspace=workspace(T, V, D))
    want, size, tokens = embed_grad(ids, d, V, -2.0)
    assert_within(grad.contiguous(), want, (tokens + 4) * E * size)
    assert not torch.signbit(grad[(tokens[:, 0] == 0).cuda()]).any()
    assert torch.isnan(held[0]).all() and torch.isnan(held[V + 1]).all()
    assert torch.isnan(held[:, :apart // 2]).all() and torch.isnan(held[:, apart // 2 + D:]).all()


# an id's frequency one over its rank, as words have it: half of the tokens are of one workgroup's ids, hundreds of them among any 256 tokens
@pytest.mark.parametrize("T,V,D", [(60_001, 70_001, 16), (20_000, 65_536, 24), (9_000, 257, 40)])
def test_gradient_of_words(T, V, D):
    g = torch.Generator().manual_seed(T)
    ids = ((V + 1.0) ** torch.rand(T, generator=g, dtype=torch.float64)).int() - 1
    ids[torch.rand(T, generator=g) < 0.03] = -1
    d = random(5, T, D, dtype=torch.bfloat16)
    grad, ws = filled(torch.float32, V, D), workspace(T, V, D)
    binding.sgap_embed_grad(T, V, D, ids.cuda(), d.cuda(), grad, workspace=ws)
    want, size, tokens = embed_grad(ids, d, V, 1.0)
    assert_within(grad, want, (tokens + 4) * E * size)


@pytest.mark.parametrize("others", OTHERS)
@pytest.mark.parametrize("dtype,grad_dtype", [(torch.float32, torch.float32), (torch.float16, torch.float16), (torch.bfloat16, torch.float32)])
@pytest.mark.parametrize("T,V,D,kind", [(1, 5, 3, "uniform"), (100, 30, 77, "mixed"), (500, 12, 1001, "skewed"), (333, 1000, 136, "skewed"), (90, 7, 64, "none")])
def test_gradient_is_added(T, V, D, kind, dtype, grad_dtype, others):
    ids, d = among(others, draw_ids(kind, T, V), random(1, T, D, dtype=dtype))
    was = random(2, V, D, dtype=grad_dtype)
    grad = was.cuda()
    binding.sgap_embed_grad(len(ids), V, D, ids.cuda(), d.cuda(), grad, scale=-1.5, accumulate=True, workspace=workspace(len(ids), V, D))
    want, size, tokens = embed_grad(ids, d, V, -1.5)
    none = (tokens[:, 0] == 0)
    assert torch.equal(grad.cpu()[none], was[none])
    assert_within(grad, want + was.double(), (tokens + 5) * E * (size + was.double().abs()))


def test_gradient_of_no_tokens_clears_the_table():
    grad = filled(torch.bfloat16, 50, 33)
    binding.sgap_embed_grad(0, 50, 33, torch.empty(0, dtype=torch.int32, device="cuda"), torch.empty(0, 33, dtype=torch.bfloat16, device="cuda"), grad,
                            workspace=workspace(0, 50, 33))
    assert torch.equal(grad, torch.zeros_like(grad))


@pytest.mark.parametrize("others", OTHERS)
@pytest.mark.parametrize("grad_dtype", [torch.float32, torch.float16])
def test_gradient_with_rows_apart(grad_dtype, others):
    V, D = 37, 51
    ids, d = among(others, draw_ids("mixed", 400, V), random(1, 400, D + 9, dtype=torch.float16))
    T = len(ids)
    grad = filled(grad_dtype, V, D + 6)
    binding.sgap_embed_grad(T, V, D, ids.cuda(), d.cuda()[:, 3:3 + D], grad[:, 1:1 + D], workspace=workspace(T, V, D))
    want, size, tokens = embed_grad(ids, d[:, 3:3 + D], V, 1.0)
    assert_within(grad[:, 1:1 + D].contiguous(), want, (tokens + 4) * E * size)
    assert torch.isnan(grad[:, 0]).all() and torch.isnan(grad[:, 1 + D:]).all()


def test_gradient_against_differences():
    # <dout, embed(W + h Z) - embed(W - h Z)> / 2 h = <dW, Z>: the lookup is linear, so that differences of 64 bits are exact to rounding
    T, V, D = 60, 20, 24
    ids, d, z = draw_ids("mixed", T, V), random(1, T, D), random(2, V, D)
    grad = filled(torch.float32, V, D)
    binding.sgap_embed_grad(T, V, D, ids.cuda(), d.cuda(), grad, scale=1.25, workspace=workspace(T, V, D))
    h, w = 0.5, random(3, V, D).double()
    slope = ((embed(ids, w + h * z.double(), 1.25) - embed(ids, w - h * z.double(), 1.25)) * d.double()).sum() / (2 * h)
    _, size, tokens = embed_grad(ids, d, V, 1.25)
    assert abs((grad.cpu().double() * z.double()).sum() - slope) <= ((tokens + 6) * E * size * z.double().abs()).sum()


@pytest.mark.parametrize("T", [3_000, 9_000])
def test_the_same_bits_on_every_call(T):
    V, D = 200, 264
    ids, d = draw_ids("skewed", T, V).cuda(), random(1, T, D, dtype=torch.bfloat16).cuda()
    first = None
    for _ in range(3):
        grad, ws = filled(torch.bfloat16, V, D), workspace(T, V, D)
        binding.sgap_embed_grad(T, V, D, ids, d, grad, workspace=ws)
        first = grad if first is None else first
        assert torch.equal(grad.view(torch.int16), first.view(torch.int16))


@pytest.mark.parametrize("T", [500, 8_500])
def test_captured_and_replayed_on_other_tokens(T):
    V, D = 60, 136
    ids, d = draw_ids("skewed", T, V).cuda(), random(1, T, D).cuda()
    w, out, grad, ws = random(2, V, D).cuda(), filled(torch.float32, T, D), filled(torch.float32, V, D), workspace(T, V, D)

    def both():
        binding.sgap_embed(T, V, D, ids, w, out)
        binding.sgap_embed_grad(T, V, D, ids, d, grad, workspace=ws)

    both()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for seed in (3, 4, 5):
        ids.copy_(draw_ids("mixed", T, V, seed))
        d.copy_(random(seed, T, D))
        out.fill_(float("nan"))
        grad.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        want, size, tokens = embed_grad(ids.cpu(), d.cpu(), V, 1.0)
        assert_within(grad, want, (tokens + 4) * E * size)
        assert_within(out, embed(ids.cpu(), w.cpu(), 1.0), 0.0)


@pytest.mark.parametrize("T", [2_000, 8_500])
def test_two_streams_with_a_workspace_each(T):
    V, D = 100, 264
    streams = [torch.cuda.Stream() for _ in range(2)]
    made = []
    for i, s in enumerate(streams):
        ids, d = draw_ids("skewed", T, V, i), random(i, T, D)
        with torch.cuda.stream(s):
            made.append((ids, d, ids.cuda(), d.cuda(), filled(torch.float32, V, D), workspace(T, V, D)))
    torch.cuda.synchronize()
    for _ in range(3):
        for s, (_, _, ids, d, grad, ws) in zip(streams, made):
            binding.sgap_embed_grad(T, V, D, ids, d, grad, workspace=ws, stream=s)
    torch.cuda.synchronize()
    for ids, d, _, _, grad, _ in made:
        want, size, tokens = embed_grad(ids, d, V, 1.0)
        assert_within(grad, want, (tokens + 4) * E * size)


@pytest.mark.parametrize("others", OTHERS)
def test_places_beyond_32_bits(others):
    # a table of 4.3 GB, whose last rows lie beyond 2^32 bytes (2^31 elements), and a gradient of the same size
    V, D, T = 1 << 19, 4104, 64
    ids = torch.arange(V - T, V, dtype=torch.int32).flip(0)
    w = torch.empty(V, D, dtype=torch.float16, device="cuda")
    rows = random(1, T, D, dtype=torch.float16)
    w[V - T:] = rows.cuda()
    out = filled(torch.float16, T, D)
    binding.sgap_embed(T, V, D, ids.cuda(), w, out)
    assert torch.equal(out.cpu(), rows.flip(0))
    ids, out = among(others, ids, out.cpu())
    binding.sgap_embed_grad(len(ids), V, D, ids.cuda(), out.cuda(), w, workspace=workspace(len(ids), V, D))
    assert torch.equal(w[V - T:].cpu(), rows)
    assert not w[:V - T].any()


def test_a_short_workspace_or_another_type_is_refused():
    ids, d, w = torch.zeros(9, dtype=torch.int32, device="cuda"), torch.zeros(9, 4, device="cuda"), torch.zeros(5, 4, device="cuda")
    ws = workspace(9, 5, 4)
    with pytest.raises(binding.SgapError, match="workspace"):
        binding.sgap_embed_grad(9, 5, 4, ids, d, w)
    with pytest.raises(binding.SgapError, match="workspace"):
        binding.sgap_embed_grad(9, 5, 4, ids, d, w, workspace=ws[:-256])
    with pytest.raises(ValueError, match="ids"):
        binding.sgap_embed(8, 5, 4, ids, w, d[:8])
    with pytest.raises(TypeError, match="ids"):
        binding.sgap_embed(9, 5, 4, ids.long(), w, d)
    with pytest.raises(TypeError, match="out"):
        binding.sgap_embed(9, 5, 4, ids, w, d.half())
    with pytest.raises(binding.SgapError, match="type"):
        binding.sgap_embed_grad(9, 5, 4, ids, d, w.half(), workspace=ws)
    with pytest.raises(binding.SgapError, match="scale"):
        binding.sgap_embed(9, 5, 4, ids, w, d, scale=float("inf"))


assert U[torch.bfloat16] == 2.0**-8
