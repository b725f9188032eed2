"""What the calls around a mixture of experts (balance loss, embeddings, numbers of 8 bits) refuse before anything is launched,
through the C ABI with made-up addresses and through the binding.  No GPU."""
import pytest
import torch

from paper_2209_02882_amd import binding
from test_experts_refusals import P, refused

BALANCE = dict(T=100, E=16, k=2, S=3, dtype=0, logits=P, ld=16, experts=P, segments=P, loss=P, counts=P, rows=P, workspace=P,
               bytes=1 << 20, stream=None)
BALANCE_GRAD = dict(T=100, E=16, k=2, S=3, dtype=0, logits=P, ld=16, experts=P, segments=P, counts=P, rows=P, dloss=P, accumulate=0,
                    dlogits=P, ldd=16, stream=None)


@pytest.mark.parametrize("changes,text", [
    (dict(T=-1), "negative"), (dict(E=0), "experts"), (dict(E=1025), "experts"), (dict(k=0), "k must"), (dict(k=17), "k must"),
    (dict(E=1), "k must"), (dict(T=2**30), "int32"), (dict(S=0), "sequences"), (dict(S=65537), "sequences"),
    (dict(dtype=3), "type"), (dict(ld=15), "row"), (dict(segments=None), "segments"), (dict(logits=None), "null"),
    (dict(experts=None), "null"), (dict(counts=None), "null"), (dict(rows=None), "null"),
])
def test_balance(changes, text):
    refused("sgap_route_balance", BALANCE, text, **changes)
    refused("sgap_route_balance_grad", BALANCE_GRAD, text, **changes)


@pytest.mark.parametrize("changes,text", [
    (dict(loss=None), "null"), (dict(workspace=None), "workspace"), (dict(bytes=100), "workspace"), (dict(workspace=P + 8), "aligned"),
])
def test_balance_results(changes, text):
    refused("sgap_route_balance", BALANCE, text, **changes)


@pytest.mark.parametrize("changes,text", [
    (dict(dloss=None), "null"), (dict(dlogits=None), "null"), (dict(ldd=15), "row"), (dict(accumulate=2), "accumulate"),
])
def test_balance_gradient(changes, text):
    refused("sgap_route_balance_grad", BALANCE_GRAD, text, **changes)


EMBED = dict(T=10, V=100, D=8, dtype=2, ids=P, weights=P, ldw=8, scale=1.0, out=P, ldo=8, stream=None)
EMBED_GRAD = dict(T=10, V=100, D=8, dtype=2, ids=P, dout=P, ldo=8, scale=1.0, accumulate=0, grad_dtype=0, weights=P, ldw=8, workspace=P,
                  bytes=1 << 20, stream=None)


@pytest.mark.parametrize("changes,text", [
    (dict(T=-1), "negative"), (dict(D=-8), "negative"), (dict(V=0), "table"), (dict(V=2**31 - 1), "int32"), (dict(T=2**31 - 1), "int32"),
    (dict(dtype=4), "type"), (dict(ldw=7), "row"), (dict(ldo=7), "row"), (dict(scale=float("nan")), "scale"),
    (dict(scale=float("inf")), "scale"), (dict(ids=None), "null"), (dict(weights=None), "null"),
])
def test_embed(changes, text):
    refused("sgap_embed", EMBED, text, **changes)
    refused("sgap_embed_grad", EMBED_GRAD, text, **changes)


@pytest.mark.parametrize("changes,text", [
    (dict(dout=None), "null"), (dict(grad_dtype=1), "type"), (dict(accumulate=-1), "accumulate"), (dict(workspace=None), "workspace"),
    (dict(bytes=400), "workspace"), (dict(workspace=P + 4), "aligned"),
])
def test_embed_gradient(changes, text):
    refused("sgap_embed_grad", EMBED_GRAD, text, **changes)
    if "dout" in changes:
        refused("sgap_embed", EMBED, text, out=None)


ROWS = dict(R=10, K=100, dtype=1, X=P, ldx=100, codes=P, scales=P, stream=None)
WEIGHTS = dict(G=3, K=100, N=70, dtype=1, W=P, codes=P, scales=P, codes_t=P, scales_t=P, stream=None)


@pytest.mark.parametrize("changes,text", [
    (dict(R=-1), "negative"), (dict(K=-1), "negative"), (dict(R=2**31 - 1), "int32"), (dict(K=2**31 - 1), "int32"), (dict(dtype=-1), "type"),
    (dict(ldx=99), "ldx"), (dict(X=None), "null"), (dict(codes=None), "null"), (dict(scales=None), "null"), (dict(codes=P + 8), "aligned"),
])
def test_f8_rows(changes, text):
    refused("sgap_f8_rows", ROWS, text, **changes)


@pytest.mark.parametrize("changes,text", [
    (dict(G=0), "group"), (dict(G=2**21), "groups"), (dict(K=-1), "negative"), (dict(N=2**31 - 1), "int32"),
    (dict(G=2**20, K=2**31 - 65536, N=2**31 - 65536), "memory"), (dict(dtype=3), "type"), (dict(W=None), "null"), (dict(codes=None), "null"),
    (dict(scales=None), "null"), (dict(codes_t=None), "together"), (dict(scales_t=None), "together"), (dict(codes=P + 1), "aligned"),
    (dict(codes_t=P + 8), "aligned"),
])
def test_f8_weights(changes, text):
    refused("sgap_f8_weights", WEIGHTS, text, **changes)


MM = dict(G=4, R=100, K=16, N=24, dtype=2, offsets=P, X=P, x_scales=P, x_rows=100, src=None, src_div=1, W=P, w_scales=P, Y=P, ldy=24,
          stream=None)


@pytest.mark.parametrize("changes,text", [
    (dict(G=0), "group"), (dict(G=2**21), "groups"), (dict(R=-1), "negative"), (dict(K=-64), "negative"), (dict(N=-1), "negative"),
    (dict(R=2**31 - 1), "int32"), (dict(N=2**31 - 1), "int32"), (dict(x_rows=-1), "negative"), (dict(offsets=None), "offsets"),
    (dict(src_div=0), "src_div"), (dict(src_div=2), "src"), (dict(x_rows=99), "fewer rows"), (dict(ldy=23), "ldy"), (dict(X=None), "null"),
    (dict(x_scales=None), "null"), (dict(Y=None), "null"), (dict(W=None), "null"), (dict(w_scales=None), "null"), (dict(dtype=9), "type"),
    (dict(X=P + 4), "aligned"), (dict(W=P + 8), "aligned"),
])
def test_products(changes, text):
    refused("sgap_grouped_mm_f8", MM, text, **changes)


def test_sizes_of_workspaces():
    assert binding.sgap_route_balance_workspace_size(0, 8, 2, 1) > 0
    assert binding.sgap_embed_grad_workspace_size(0, 1, 0) >= 8
    # start, key and order, and two rows of floats for each of 64 tiles of four times 8 tokens
    assert binding.sgap_embed_grad_workspace_size(2048, 1000, 64) == 4096 + 8192 + 8192 + 64 * 2 * 64 * 4
    # 256 tiles at most, or 2^19 numbers, however many the tokens
    assert binding.sgap_embed_grad_workspace_size(1 << 20, 1, 256) == 256 + 2 * (4 << 20) + 2048 * 2 * 256 * 4
    assert binding.sgap_embed_grad_workspace_size(1 << 20, 1, 4096) == 256 + 2 * (4 << 20) + 256 * 2 * 4096 * 4
    with pytest.raises(binding.SgapError):
        binding.sgap_embed_grad_workspace_size(4, 0, 8)
    with pytest.raises(binding.SgapError):
        binding.sgap_route_balance_workspace_size(4, 8, 2, 0)


def test_empty_calls_launch_nothing():
    lib = binding.load()
    assert lib.sgap_embed(*{**EMBED, "T": 0, "ids": None, "out": None}.values()) == 0
    assert lib.sgap_embed(*{**EMBED, "D": 0, "weights": None, "out": None}.values()) == 0
    assert lib.sgap_embed_grad(*{**EMBED_GRAD, "T": 0, "accumulate": 1, "ids": None, "weights": None}.values()) == 0
    assert lib.sgap_route_balance_grad(*{**BALANCE_GRAD, "T": 0, "logits": None}.values()) == 0
    assert lib.sgap_f8_rows(*{**ROWS, "R": 0, "X": None}.values()) == 0
    assert lib.sgap_f8_weights(*{**WEIGHTS, "N": 0, "W": None}.values()) == 0
    assert lib.sgap_grouped_mm_f8(*{**MM, "R": 0, "X": None, "Y": None}.values()) == 0
    # a list of no rows has no address
    assert lib.sgap_grouped_mm_f8(*{**MM, "R": 0, "x_rows": 0, "src_div": 2, "X": None, "Y": None}.values()) == 0
    assert lib.sgap_grouped_mm(4, 0, 16, 24, 2, P, None, 16, 0, None, 2, P, 0, None, 24, None) == 0
    assert lib.sgap_grouped_mm_f8(*{**MM, "N": 0, "W": None, "Y": None}.values()) == 0


def test_binding_says_what_is_wrong():
    t, i = torch.zeros(4, 8), torch.zeros(4, dtype=torch.int32)
    with pytest.raises(TypeError, match="CUDA"):
        binding.sgap_embed(4, 4, 8, i, t, t)
    with pytest.raises(TypeError, match="float32, float16"):
        binding.sgap_embed(4, 4, 8, i, t.int(), t)
    with pytest.raises(TypeError, match="CUDA"):
        binding.sgap_embed_grad(4, 4, 8, i, t, t)
    with pytest.raises(TypeError, match="CUDA"):
        binding.sgap_route_balance(4, 8, 2, 1, t, i, None, t, i, i)
    with pytest.raises(TypeError, match="CUDA"):
        binding.sgap_f8_rows(4, 8, t, t, t)
    with pytest.raises(TypeError, match="CUDA"):
        binding.sgap_f8_weights(1, 8, 4, t, t, t)
    with pytest.raises(ValueError, match="matrix of codes"):
        binding.sgap_grouped_mm_f8(1, 4, 8, 4, None, t[0], t, t, t, t)
