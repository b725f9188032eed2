"""A mixture-of-experts layer out of the library's calls, as one would train it and serve it.

Training: the router gives every token k experts, the tokens' rows are multiplied by their experts' weights without being
copied into order first, and the experts' rows are summed up by token; the gradients go the same way back.  A balance loss keeps
the experts evenly used, an embedding makes rows of tokens, and the products may go in 8 bits.  Serving: the same with the
experts' weights in 4 or 8 bits.

    python -m paper_2209_02882_amd.experts          trains a small layer for a few steps, then serves it in 16, 8 and 4 bits, and
                                                    trains a small model of tokens in 8 bits

The activation between the two products and the products without experts are torch's; everything that goes by expert or by
token's number is the library's.  The gradients are not
differentiable themselves: a second derivative raises an error.
"""
from __future__ import annotations

import torch
from torch.autograd.function import once_differentiable

from . import binding


class Route(torch.autograd.Function):
    """(gates, slot, order, offsets) of logits T x E; only the gates have a gradient."""

    @staticmethod
    def forward(ctx, logits, k):
        T, E = logits.shape
        dev = logits.device
        gates = torch.empty((T, k), device=dev)
        experts, slot = (torch.empty((T, k), dtype=torch.int32, device=dev) for _ in range(2))
        order = torch.empty(T * k, dtype=torch.int32, device=dev)
        offsets = torch.empty(E + 1, dtype=torch.int32, device=dev)
        workspace = torch.empty(binding.sgap_route_topk_workspace_size(T, E, k), dtype=torch.uint8, device=dev)
        binding.sgap_route_topk(T, E, k, logits, gates, experts, slot, order, offsets, workspace=workspace)
        ctx.save_for_backward(logits, gates, experts)
        ctx.mark_non_differentiable(slot, order, offsets)
        return gates, slot, order, offsets

    @staticmethod
    @once_differentiable
    def backward(ctx, dgates, *_):
        logits, gates, experts = ctx.saved_tensors
        T, E = logits.shape
        dlogits = torch.empty_like(logits)
        binding.sgap_route_topk_grad(T, E, gates.shape[1], logits, gates, experts, dgates.contiguous(), dlogits)
        return dlogits, None


class RouteBalanced(torch.autograd.Function):
    """(gates, slot, order, offsets, loss, counts) of logits T x E: Route with the balance loss over the sequences that `segments`
    says (None: one of all tokens), a float, and each sequence's pairs by expert.  The gates and the loss have gradients, which
    meet in the logits without an array between them."""

    @staticmethod
    def forward(ctx, logits, k, segments):
        T, E = logits.shape
        S = 1 if segments is None else segments.numel() - 1
        dev = logits.device
        gates, loss = torch.empty((T, k), device=dev), torch.empty(1, device=dev)
        experts, slot = (torch.empty((T, k), dtype=torch.int32, device=dev) for _ in range(2))
        order = torch.empty(T * k, dtype=torch.int32, device=dev)
        offsets = torch.empty(E + 1, dtype=torch.int32, device=dev)
        counts, rows = torch.empty((S, E), dtype=torch.int32, device=dev), torch.empty(S, dtype=torch.int32, device=dev)
        size = max(binding.sgap_route_topk_workspace_size(T, E, k), binding.sgap_route_balance_workspace_size(T, E, k, S))
        workspace = torch.empty(size, dtype=torch.uint8, device=dev)
        binding.sgap_route_topk(T, E, k, logits, gates, experts, slot, order, offsets, workspace=workspace)
        binding.sgap_route_balance(T, E, k, S, logits, experts, segments, loss, counts, rows, workspace=workspace)
        ctx.save_for_backward(logits, gates, experts, segments, counts, rows)
        ctx.mark_non_differentiable(slot, order, offsets, counts)
        return gates, slot, order, offsets, loss[0], counts

    @staticmethod
    @once_differentiable
    def backward(ctx, dgates, _slot, _order, _offsets, dloss, _counts):
        logits, gates, experts, segments, counts, rows = ctx.saved_tensors
        T, E = logits.shape
        k, S = gates.shape[1], counts.shape[0]
        dlogits = torch.empty_like(logits)
        binding.sgap_route_topk_grad(T, E, k, logits, gates, experts, dgates.contiguous(), dlogits)
        binding.sgap_route_balance_grad(T, E, k, S, logits, experts, segments, counts, rows, dloss.float().reshape(1), dlogits,
                                        accumulate=True)
        return dlogits, None, None


class Embed(torch.autograd.Function):
    """Rows of weights (V x D) times scale by token; zeros for a token outside the table."""

    @staticmethod
    def forward(ctx, ids, weights, scale):
        V, D = weights.shape
        out = torch.empty((ids.numel(), D), dtype=weights.dtype, device=weights.device)
        binding.sgap_embed(ids.numel(), V, D, ids, weights, out, scale=scale)
        ctx.save_for_backward(ids)
        ctx.V, ctx.scale = V, scale
        return out

    @staticmethod
    @once_differentiable
    def backward(ctx, dout):
        (ids,) = ctx.saved_tensors
        T, D = dout.shape
        dweights = torch.empty((ctx.V, D), dtype=dout.dtype, device=dout.device)
        workspace = torch.empty(binding.sgap_embed_grad_workspace_size(T, ctx.V, D), dtype=torch.uint8, device=dout.device)
        binding.sgap_embed_grad(T, ctx.V, D, ids, dout.contiguous(), dweights, scale=ctx.scale, workspace=workspace)
        return None, dweights, None


class Embedding(torch.nn.Module):
    """ids (int32, any shape) -> scale * their rows of the table."""

    def __init__(self, vocabulary, width, scale=1.0, dtype=torch.bfloat16, device="cuda"):
        super().__init__()
        self.scale = float(scale)
        self.weights = torch.nn.Parameter((torch.randn(vocabulary, width, device=device) * width ** -0.5).to(dtype))

    def forward(self, ids):
        return Embed.apply(ids.reshape(-1).contiguous(), self.weights, self.scale).view(*ids.shape, self.weights.shape[1])


class GroupedMM(torch.autograd.Function):
    """Rows of x times their expert's weights (E x N x K).  Where they are `gathered`, x has the tokens' rows, row r is
    x[order[r] // k], and the gradient of x is the sum over a token's rows; else x lies in order already."""

    @staticmethod
    def forward(ctx, x, weights, offsets, order, slot, gathered):
        G, N, K = weights.shape
        k = slot.shape[1]
        R = order.numel()
        y = torch.empty((R, N), dtype=x.dtype, device=x.device)
        gather = {"src": order, "src_div": k} if gathered else {}
        binding.sgap_grouped_mm(G, R, K, N, offsets, x, weights, y, "nk", **gather)
        ctx.save_for_backward(x, weights, offsets, order, slot)
        ctx.gather = gather
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        x, weights, offsets, order, slot = ctx.saved_tensors
        G, N, K = weights.shape
        R, dy = order.numel(), dy.contiguous()
        dx = dw = None
        if ctx.needs_input_grad[0]:
            dx = torch.empty((R, K), dtype=x.dtype, device=x.device)
            binding.sgap_grouped_mm(G, R, N, K, offsets, dy, weights, dx, "kn")
            # a pair's row is rounded to x's type, in which the product stores it, and once more the sum of a token's k rows:
            # half the bytes written and read that rows of floats would be
            if ctx.gather:
                rows, dx = dx, torch.empty_like(x)
                binding.sgap_route_combine(slot.shape[0], slot.shape[1], K, rows, slot, None, dx)
        if ctx.needs_input_grad[1]:
            dw = torch.empty_like(weights)
            binding.sgap_grouped_mm_wgrad(G, R, K, N, offsets, x, dy, dw, "nk", **ctx.gather)
        return dx, dw, None, None, None, None


def blocks8(n):
    return -(-n // binding.SGAP_F8_BLOCK)


def codes8(*shape, device):
    return torch.empty(shape, dtype=torch.uint8, device=device).view(torch.float8_e4m3fn)


def rows8(x):
    """(codes, scales) in 8 bits of the rows of x."""
    R, K = x.shape
    codes, scales = codes8(R, blocks8(K) * binding.SGAP_F8_BLOCK, device=x.device), torch.empty((R, blocks8(K)), device=x.device)
    binding.sgap_f8_rows(R, K, x, codes, scales)
    return codes, scales


class Weights8:
    """Weights E x N x K in 8 bits; `both`: transposed too, as the gradient of the rows wants them."""

    def __init__(self, weights, both=False):
        self.shape = E, N, K = weights.shape
        dev, block = weights.device, binding.SGAP_F8_BLOCK
        self.codes, self.scales = codes8(E, N, blocks8(K) * block, device=dev), torch.empty((E, blocks8(N), blocks8(K)), device=dev)
        self.codes_t = self.scales_t = None
        if both:
            self.codes_t, self.scales_t = codes8(E, K, blocks8(N) * block, device=dev), torch.empty((E, blocks8(K), blocks8(N)), device=dev)
        binding.sgap_f8_weights(E, K, N, weights, self.codes, self.scales, self.codes_t, self.scales_t)

    def rows(self, x, offsets, R, **gather):
        E, N, K = self.shape
        y = torch.empty((R, N), dtype=x.dtype, device=x.device)
        binding.sgap_grouped_mm_f8(E, R, K, N, offsets, *rows8(x), self.codes, self.scales, y, **gather)
        return y


class GroupedMM8(torch.autograd.Function):
    """GroupedMM with rows and weights in 8 bits, and the gradient of the rows too.  The weights' gradient is GroupedMM's: its inner
    dimension is a group's rows, and what blocks of them would have to be cut in no call knows beforehand."""

    @staticmethod
    def forward(ctx, x, weights, offsets, order, slot, gathered):
        # the transposed codes wait for the backward pass where there will be one
        held = Weights8(weights, both=ctx.needs_input_grad[0])
        ctx.gather = {"src": order, "src_div": slot.shape[1]} if gathered else {}
        ctx.save_for_backward(x, weights, offsets, order, slot, held.codes_t, held.scales_t)
        return held.rows(x, offsets, order.numel(), **ctx.gather)

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        x, weights, offsets, order, slot, codes_t, scales_t = ctx.saved_tensors
        G, N, K = weights.shape
        R, dy = order.numel(), dy.contiguous()
        dx = dw = None
        if ctx.needs_input_grad[0]:
            dx = torch.empty((R, K), dtype=x.dtype, device=x.device)
            binding.sgap_grouped_mm_f8(G, R, N, K, offsets, *rows8(dy), codes_t, scales_t, dx)
            if ctx.gather:
                rows, dx = dx, torch.empty_like(x)
                binding.sgap_route_combine(slot.shape[0], slot.shape[1], K, rows, slot, None, dx)
        if ctx.needs_input_grad[1]:
            dw = torch.empty_like(weights)
            binding.sgap_grouped_mm_wgrad(G, R, K, N, offsets, x, dy, dw, "nk", **ctx.gather)
        return dx, dw, None, None, None, None


class Combine(torch.autograd.Function):
    """The experts' rows summed up by token, each times its gate."""

    @staticmethod
    def forward(ctx, rows, gates, slot, order):
        T, k = slot.shape
        out = torch.empty((T, rows.shape[1]), dtype=rows.dtype, device=rows.device)
        binding.sgap_route_combine(T, k, rows.shape[1], rows, slot, gates, out)
        ctx.save_for_backward(rows, gates, slot, order)
        return out

    @staticmethod
    @once_differentiable
    def backward(ctx, dout):
        rows, gates, slot, order = ctx.saved_tensors
        T, k = slot.shape
        drows, dgates = torch.empty_like(rows), torch.empty_like(gates)
        binding.sgap_route_combine_grad(T, k, rows.shape[1], rows, slot, order, gates, dout.contiguous(), drows, dgates)
        return drows, dgates, None, None


def gated(h):
    """silu of the first half of the columns times the second."""
    a, b = h.chunk(2, dim=1)
    return torch.nn.functional.silu(a) * b


def quantise(weights, group_k):
    """(codes, scales, zeros) in 4 bits of weights E x N x K: group_k neighbours along K share a scale and a zero point."""
    E, N, K = weights.shape
    w = weights.float().view(E, N, K // group_k, group_k)
    low, high = w.amin(3).clamp(max=0), w.amax(3).clamp(min=0)
    scales = ((high - low) / 15).clamp(min=1e-8).to(weights.dtype)
    zeros = (-low / scales.float()).round().clamp(0, 15)
    codes = (w / scales.float()[..., None] + zeros[..., None]).round().clamp(0, 15).view(E, N, K).to(torch.uint8)
    return codes[..., 0::2] | (codes[..., 1::2] << 4), scales, zeros.to(torch.uint8)


class Weights4:
    """Weights E x N x K in 4 bits, laid out once for sgap_grouped_mm_w4."""

    def __init__(self, weights, group_k=64):
        self.shape, self.group_k = weights.shape, group_k
        E, N, K = weights.shape
        codes, scales, zeros = quantise(weights, group_k)
        size = binding.sgap_w4_layout_size(E, K, N, group_k, zeros=True)
        self.data = torch.empty(size, dtype=torch.uint8, device=weights.device)
        binding.sgap_w4_layout(E, K, N, group_k, codes.contiguous(), scales, zeros, self.data)

    def rows(self, x, offsets, R, **gather):
        E, N, K = self.shape
        y = torch.empty((R, N), dtype=x.dtype, device=x.device)
        binding.sgap_grouped_mm_w4(E, R, K, N, self.group_k, offsets, x, self.data, y, zeros=True, **gather)
        return y


class ExpertLayer(torch.nn.Module):
    """x (T x width) -> sum over each token's k experts of gate * down(gated(up(x)))."""

    def __init__(self, width, hidden, experts, k, dtype=torch.bfloat16, device="cuda", eight_bits=False):
        """eight_bits: the experts' products, and the gradients of their rows, go in 8 bits."""
        super().__init__()
        self.k, self.product = k, GroupedMM8 if eight_bits else GroupedMM
        new = lambda *shape: torch.nn.Parameter((torch.randn(shape, device=device) * shape[-1] ** -0.5).to(dtype))  # noqa: E731
        self.router, self.up, self.down = new(experts, width), new(experts, 2 * hidden, width), new(experts, width, hidden)
        self.served = None

    def logits(self, x):
        """In 32 bits: in 16, experts within half a unit of one another would be equal, and the first of them chosen."""
        return x.float() @ self.router.float().t()

    def by_expert(self, x, gates, slot, order, offsets):
        h = gated(self.product.apply(x, self.up, offsets, order, slot, True))
        return Combine.apply(self.product.apply(h, self.down, offsets, order, slot, False), gates, slot, order)

    def forward(self, x):
        return self.by_expert(x, *Route.apply(self.logits(x), self.k))

    def balanced(self, x, segments=None):
        """(what forward gives, the balance loss, pairs of each sequence and expert); segments: S + 1 ends of packed sequences."""
        *routed, loss, counts = RouteBalanced.apply(self.logits(x), self.k, segments)
        return self.by_expert(x, *routed), loss, counts

    @torch.no_grad()
    def quantise(self, group_k=64, bits=4):
        """From now on serve() has the experts as they are now, in 4 bits (or 8, without regard to group_k); after further training,
        quantise again."""
        if bits not in (4, 8):
            raise ValueError("bits must be 4 or 8")
        self.served = tuple(Weights4(w, group_k) if bits == 4 else Weights8(w) for w in (self.up, self.down))

    @torch.no_grad()
    def serve(self, x):
        if self.served is None:
            return self(x)
        up, down = self.served
        gates, slot, order, offsets = Route.apply(self.logits(x), self.k)
        R = order.numel()
        h = gated(up.rows(x, offsets, R, src=order, src_div=self.k))
        out = torch.empty_like(x)
        binding.sgap_route_combine(x.shape[0], self.k, x.shape[1], down.rows(h, offsets, R), slot, gates, out)
        return out


def main(steps=30, tokens=512, width=256, hidden=128, experts=8, k=2):
    torch.manual_seed(0)
    layer = ExpertLayer(width, hidden, experts, k)
    wanted = torch.randn(width, width, device="cuda") * width ** -0.5
    optimiser = torch.optim.Adam(layer.parameters(), lr=5e-3)
    x = torch.randn(tokens, width, device="cuda").bfloat16()
    losses = []
    for step in range(steps):
        loss = (layer(x).float() - x.float() @ wanted).square().mean()
        optimiser.zero_grad()
        loss.backward()
        optimiser.step()
        losses.append(loss.item())
        if step % 10 == 0 or step == steps - 1:
            print(f"step {step:3d}: loss {losses[-1]:.4f}", flush=True)
    x = torch.randn(4, width, device="cuda").bfloat16()
    full = layer.serve(x).float()
    for bits in (8, 4):
        layer.quantise(bits=bits)
        off = (layer.serve(x).float() - full).norm() / full.norm()
        print(f"4 tokens served with the experts in {bits} bits: {100 * off.item():.1f}% off the 16-bit ones")
    return losses, off.item()


class TokenModel(torch.nn.Module):
    """ids (T) -> (logits T x vocabulary of the next ones, balance loss): an embedding, one layer of experts beside it, and the
    embedding's rows again as weights of the result."""

    def __init__(self, vocabulary, width, hidden, experts, k, dtype=torch.bfloat16, device="cuda", eight_bits=True):
        super().__init__()
        self.embedding = Embedding(vocabulary, width, width ** 0.5, dtype, device)
        self.layer = ExpertLayer(width, hidden, experts, k, dtype, device, eight_bits)

    def forward(self, ids, segments=None):
        x = self.embedding(ids)
        out, balance, _ = self.layer.balanced(x, segments)
        return (x + out) @ self.embedding.weights.t(), balance


def train_tokens(steps=30, vocabulary=500, lengths=(200, 1, 311), width=128, hidden=128, experts=8, k=2):
    """A few steps on packed sequences whose next token follows from the last one."""
    torch.manual_seed(0)
    model = TokenModel(vocabulary, width, hidden, experts, k)
    optimiser = torch.optim.Adam(model.parameters(), lr=3e-3)
    ids = torch.randint(0, vocabulary, (sum(lengths),), device="cuda", dtype=torch.int32)
    follows = torch.randperm(vocabulary, device="cuda")
    segments = torch.tensor([0, *lengths], device="cuda").cumsum(0).int()
    losses = []
    for step in range(steps):
        logits, balance = model(ids, segments)
        loss = torch.nn.functional.cross_entropy(logits.float(), follows[ids.long()])
        optimiser.zero_grad()
        (loss + 0.01 * balance).backward()
        optimiser.step()
        losses.append(loss.item())
        if step % 10 == 0 or step == steps - 1:
            print(f"step {step:3d}: loss {losses[-1]:.4f}, balance {balance.item():.3f}", flush=True)
    return losses


if __name__ == "__main__":
    main()
    train_tokens()
