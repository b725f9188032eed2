"""The layer that puts the calls together: its gradients against autograd of a plain layer, its training and its serving."""
import pytest
import torch

from paper_2209_02882_amd import experts

pytestmark = pytest.mark.gpu


def plain(layer, x):
    """The same layer in 64 bits, one expert after the other."""
    logits = x @ layer.router.double().t()
    top, chosen = torch.topk(logits, layer.k, dim=1)
    gates = torch.softmax(top, dim=1)
    out = torch.zeros_like(x)
    for e in range(layer.up.shape[0]):
        h = experts.gated(x @ layer.up[e].double().t()) @ layer.down[e].double().t()
        out = out + h * torch.where(chosen == e, gates, torch.zeros_like(gates)).sum(1, keepdim=True)
    return out


@pytest.mark.parametrize("tokens,width,hidden,n,k", [(100, 64, 48, 6, 2), (33, 40, 24, 5, 1), (70, 33, 17, 4, 4)])
def test_gradients_of_the_layer(tokens, width, hidden, n, k):
    torch.manual_seed(tokens)
    layer = experts.ExpertLayer(width, hidden, n, k, dtype=torch.float32)
    x = torch.randn(tokens, width, device="cuda", requires_grad=True)
    weight = torch.randn(tokens, width, device="cuda")
    out = layer(x)
    (out * weight).sum().backward()
    got = [x.grad] + [p.grad for p in (layer.router, layer.up, layer.down)]
    x64 = x.detach().double().requires_grad_()
    params = [p.detach().double().requires_grad_() for p in (layer.router, layer.up, layer.down)]
    twin = experts.ExpertLayer(width, hidden, n, k, dtype=torch.float32)
    twin.router, twin.up, twin.down = (torch.nn.Parameter(p) for p in params)
    want_out = plain(twin, x64)
    (want_out * weight.double()).sum().backward()
    want = [x64.grad, twin.router.grad, twin.up.grad, twin.down.grad]
    # chains of at most 4 sums of under 256 products: 2^-23 * 256 * 4 of the largest value, with room for the activation
    assert (out.double() - want_out).abs().max() <= 2.0**-12 * want_out.abs().max()
    for g, w in zip(got, want):
        assert (g.double() - w).abs().max() <= 2.0**-12 * w.abs().max()


def test_the_example_learns_and_serves():
    losses, off = experts.main(steps=20)
    assert losses[-1] < 0.8 * losses[0]
    # a step of 4 bits is a fifteenth of a group's range: an error of 1/52 of it in the mean square, where the range of 64
    # normal values is about 4.7 of their deviation: 9 % of a weight, and the layer has two of them
    assert off < 0.25


def test_serving_in_16_bits_is_the_layer():
    torch.manual_seed(1)
    layer = experts.ExpertLayer(64, 32, 4, 2)
    x = torch.randn(9, 64, device="cuda").bfloat16()
    assert torch.equal(layer.serve(x), layer(x))
