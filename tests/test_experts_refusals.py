"""What the calls of a mixture of experts refuse before anything is launched, through the C ABI with made-up addresses and
through the binding.  No GPU."""
import pytest
import torch

from paper_2209_02882_amd import binding

BAD = binding.SGAP_ERR_INVALID_ARG
P = 0x10000  # stands for a device pointer: refused calls never use it


def refused(name, args, text, **changes):
    values = dict(args)
    for key, value in changes.items():
        assert key in values
        values[key] = value
    lib = binding.load()
    assert getattr(lib, name)(*values.values()) == BAD, changes
    assert text in lib.sgap_last_error().decode(), (changes, lib.sgap_last_error())


ROUTE = dict(T=100, E=16, k=2, dtype=0, logits=P, ld=16, renormalise=1, gates=P, experts=P, slot=P, order=P, offsets=P,
             workspace=P, bytes=1 << 20, stream=None)


@pytest.mark.parametrize("changes,text", [
    (dict(T=-1), "negative"), (dict(E=0), "experts"), (dict(E=1025), "experts"), (dict(k=0), "k must"), (dict(k=17), "k must"),
    (dict(k=5, E=4, ld=16), "k must"), (dict(T=2**31 - 1), "int32"), (dict(dtype=3), "type"), (dict(dtype=-1), "type"),
    (dict(ld=15), "ld_logits"), (dict(renormalise=2), "renormalise"), (dict(logits=None), "null"), (dict(gates=None), "null"),
    (dict(experts=None), "null"), (dict(slot=None), "null"), (dict(order=None), "null"), (dict(offsets=None), "null"),
    (dict(workspace=None), "workspace"), (dict(bytes=4), "workspace"), (dict(workspace=P + 4), "aligned"),
])
def test_route_topk(changes, text):
    refused("sgap_route_topk", ROUTE, text, **changes)


def test_route_topk_workspace_size():
    assert binding.sgap_route_topk_workspace_size(64, 1024, 16) == 0
    assert binding.sgap_route_topk_workspace_size(65, 8, 2) > 0
    with pytest.raises(binding.SgapError):
        binding.sgap_route_topk_workspace_size(10, 4, 5)


GRAD = dict(T=100, E=16, k=2, dtype=1, logits=P, ld=16, renormalise=0, gates=P, experts=P, dgates=P, dlogits=P, ldd=16, stream=None)


@pytest.mark.parametrize("changes,text", [
    (dict(T=-1), "negative"), (dict(k=0), "k must"), (dict(dtype=7), "type"), (dict(ld=3), "row"), (dict(ldd=3), "row"),
    (dict(renormalise=-1), "renormalise"), (dict(logits=None), "null"), (dict(gates=None), "null"), (dict(experts=None), "null"),
    (dict(dgates=None), "null"), (dict(dlogits=None), "null"),
])
def test_route_topk_grad(changes, text):
    refused("sgap_route_topk_grad", GRAD, text, **changes)


COMBINE = dict(T=10, k=2, D=8, dtype=2, Z=P, slot=P, gates=P, out=P, stream=None)
COMBINE_GRAD = dict(T=10, k=2, D=8, dtype=2, Z=P, slot=P, order=P, gates=P, dout=P, dZ=P, dgates=P, stream=None)


@pytest.mark.parametrize("changes,text", [
    (dict(T=-1), "negative"), (dict(D=-1), "negative"), (dict(k=0), "k must"), (dict(k=17), "k must"), (dict(T=2**30, k=4), "int32"),
    (dict(dtype=5), "type"), (dict(Z=None), "null"), (dict(slot=None), "null"),
])
def test_combine(changes, text):
    refused("sgap_route_combine", COMBINE, text, **changes)
    refused("sgap_route_combine_grad", COMBINE_GRAD, text, **changes)


@pytest.mark.parametrize("name", ["order", "gates", "dout", "dZ", "dgates"])
def test_combine_grad_needs_its_arrays(name):
    refused("sgap_route_combine_grad", COMBINE_GRAD, "null", **{name: None})


MM = dict(G=4, R=100, K=16, N=24, dtype=2, offsets=P, X=P, ldx=16, x_rows=100, src=None, src_div=1, W=P, layout=0, Y=P, ldy=24,
          stream=None)
WGRAD = dict(G=4, R=100, K=16, N=24, dtype=2, offsets=P, X=P, ldx=16, x_rows=100, src=None, src_div=1, Y=P, ldy=24, W=P, layout=0,
             stream=None)
W4 = dict(G=4, R=100, K=128, N=24, dtype=2, group_k=64, zeros=0, offsets=P, X=P, ldx=128, x_rows=100, src=None, src_div=1, W=P,
          bytes=1 << 20, Y=P, ldy=24, stream=None)


@pytest.mark.parametrize("name,args", [("sgap_grouped_mm", MM), ("sgap_grouped_mm_wgrad", WGRAD), ("sgap_grouped_mm_w4", W4)])
@pytest.mark.parametrize("changes,text", [
    (dict(G=0), "group"), (dict(G=2**21), "groups"), (dict(R=-1), "negative"), (dict(K=-64), "negative"), (dict(N=-1), "negative"),
    (dict(R=2**31 - 1), "int32"), (dict(N=2**31 - 1), "int32"), (dict(x_rows=-1), "negative"), (dict(offsets=None), "offsets"),
    (dict(src_div=0), "src_div"), (dict(src_div=2), "src"), (dict(x_rows=99), "fewer rows"), (dict(ldx=15), "ldx"),
    (dict(ldy=23), "ldy"), (dict(X=None), "null"), (dict(Y=None), "null"), (dict(W=None), "null"), (dict(dtype=9), "type"),
])
def test_products(name, args, changes, text):
    refused(name, args, text, **changes)


@pytest.mark.parametrize("name,args", [("sgap_grouped_mm", MM), ("sgap_grouped_mm_wgrad", WGRAD)])
def test_products_layout(name, args):
    refused(name, args, "layout", layout=2)


@pytest.mark.parametrize("changes,text", [
    (dict(group_k=16), "group_k"), (dict(group_k=96), "group_k"), (dict(group_k=192), "group_k"), (dict(group_k=0), "group_k"),
    (dict(group_k=256), "multiple"), (dict(K=96, ldx=128), "multiple"), (dict(zeros=2), "zeros"), (dict(dtype=0), "16-bit"),
    (dict(bytes=100), "smaller"), (dict(W=P + 8), "aligned"),
])
def test_w4(changes, text):
    refused("sgap_grouped_mm_w4", W4, text, **changes)


def test_w4_layout():
    args = dict(G=2, K=128, N=20, group_k=32, codes=P, scales=P, zeros=P, weights=P, bytes=1 << 20, stream=None)
    for changes, text in [(dict(G=0), "group"), (dict(group_k=33), "group_k"), (dict(K=100), "multiple"), (dict(bytes=10), "smaller"),
                          (dict(codes=None), "null"), (dict(scales=None), "null"), (dict(weights=None), "null"),
                          (dict(weights=P + 1), "aligned")]:
        refused("sgap_w4_layout", args, text, **changes)
    # two groups, two tiles of 16 columns, a block of 128 values: codes, then scales, then zero points
    size = binding.sgap_w4_layout_size(2, 128, 20, 32)
    assert size == 2 * 2 * 1024 + 2 * 2 * 4 * 16 * 2
    assert binding.sgap_w4_layout_size(2, 128, 20, 32, zeros=True) == size + 2 * 2 * 4 * 16
    with pytest.raises(binding.SgapError):
        binding.sgap_w4_layout_size(2, 100, 20, 32)


def test_empty_calls_launch_nothing():
    lib = binding.load()
    assert lib.sgap_grouped_mm(*{**MM, "R": 0, "X": None, "Y": None}.values()) == 0
    assert lib.sgap_grouped_mm(*{**MM, "N": 0, "W": None, "Y": None}.values()) == 0
    assert lib.sgap_grouped_mm_w4(*{**W4, "R": 0}.values()) == 0
    assert lib.sgap_route_combine(*{**COMBINE, "T": 0, "Z": None}.values()) == 0
    assert lib.sgap_route_topk_grad(*{**GRAD, "T": 0, "logits": None}.values()) == 0


def test_binding_says_what_is_wrong():
    t = torch.zeros(4, 8)
    with pytest.raises(TypeError, match="CUDA"):
        binding.sgap_grouped_mm(1, 4, 8, 8, None, t, torch.zeros(1, 8, 8), t)
    with pytest.raises(TypeError, match="float"):
        binding.sgap_grouped_mm(1, 4, 8, 8, None, t.int(), t, t)
    with pytest.raises(TypeError, match="CUDA"):
        binding.sgap_route_topk(4, 8, 2, t, t, t, t, t, t)
    with pytest.raises(TypeError, match="16"):
        binding.sgap_w4_layout(1, 32, 8, 32, t, t, None, t)
