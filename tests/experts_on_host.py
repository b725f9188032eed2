"""The calls that the layer of experts makes, on host tensors in torch's own operations, each noted by its name: for what is to
be said of the layer itself, without a GPU."""
import torch

from paper_2209_02882_amd import binding


class Calls(list):
    """In the binding's place; a list of the names of the calls that were made."""

    def __getattr__(self, name):
        if not name.startswith("sgap_"):
            raise AttributeError(name)
        if name == "sgap_route_topk_workspace_size":
            return lambda *args: 0
        step = globals()[name[len("sgap_"):]]

        def call(*args, **kwargs):
            self.append(name)
            with torch.no_grad():
                step(*args, **kwargs)

        return call


def on_host(monkeypatch):
    """The calls of the binding that a layer makes from here on."""
    from paper_2209_02882_amd import experts

    calls = Calls()
    monkeypatch.setattr(experts, "binding", calls)
    return calls


assert all(hasattr(binding, "sgap_" + name) for name in ("route_topk", "route_topk_grad", "grouped_mm", "grouped_mm_wgrad",
                                                         "route_combine", "route_combine_grad"))


def route_topk(T, E, k, logits, gates, experts, slot, order, offsets, renormalise=True, workspace=None):
    top, chosen = torch.sort(logits.double(), dim=1, descending=True, stable=True)
    gates.copy_(torch.softmax(top[:, :k], dim=1))
    experts.copy_(chosen[:, :k])
    order.copy_(torch.sort(experts.reshape(-1), stable=True)[1])
    slot.view(-1)[order.long()] = torch.arange(T * k, dtype=torch.int32)
    offsets.zero_()
    offsets[1:] = torch.cumsum(torch.bincount(experts.reshape(-1), minlength=E), 0)


def route_topk_grad(T, E, k, logits, gates, experts, dgates, dlogits, renormalise=True):
    inner = (gates * dgates).sum(1, keepdim=True)
    dlogits.zero_().scatter_(1, experts.long(), gates * (dgates - inner))


def rows_of(X, R, src, src_div):
    return X if src is None else X[torch.div(src.long(), src_div, rounding_mode="floor")]


def grouped_mm(G, R, K, N, offsets, X, W, Y, layout="nk", src=None, src_div=1):
    x = rows_of(X, R, src, src_div)
    for g in range(G):
        a, b = int(offsets[g]), int(offsets[g + 1])
        Y[a:b] = x[a:b] @ (W[g].t() if layout == "nk" else W[g])


def grouped_mm_wgrad(G, R, K, N, offsets, X, dY, dW, layout="nk", src=None, src_div=1):
    x = rows_of(X, R, src, src_div)
    for g in range(G):
        a, b = int(offsets[g]), int(offsets[g + 1])
        dW[g] = dY[a:b].t() @ x[a:b]


def route_combine(T, k, D, Z, slot, gates, out):
    z = Z[slot.long()]
    out.copy_((z if gates is None else z * gates.unsqueeze(2).to(z.dtype)).sum(1))


def route_combine_grad(T, k, D, Z, slot, order, gates, dout, dZ, dgates):
    dZ[slot.long()] = (gates.unsqueeze(2) * dout.unsqueeze(1)).to(dZ.dtype)
    dgates.copy_((Z[slot.long()] * dout.unsqueeze(1)).sum(2))
