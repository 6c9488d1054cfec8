"""A mixture-of-experts layer around the exchange, for serving and for training.

serve(): P ranks (P buffers on one GPU) with E / P experts each. Every rank routes its tokens, orders
their rows by expert as 8-bit codes and counts them for every rank; AllToAllvDynamic takes the codes and
their scales to the experts with those counts, on the device; the experts multiply them (gate and up,
then down, in 8 bits); the rows come back with the same counts, and each token's are added up, weighted.
Nothing waits for the host between the router and the result.

train(): the same layer's forward and backward pass on one rank, with experts in the tokens' own type, as
torch.autograd functions over the operators.

    python examples/moe_layer.py            # both, checked against the layer in 32 bits
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2608_00358_amd as H  # noqa: E402


def quantize_weights(w):
    """Weights (experts, columns, inner) to 8-bit codes with a scale for every expert's column."""
    scale = w.abs().amax(2).clamp_(min=1e-12) / 127.0
    return torch.round(w / scale[..., None]).to(torch.int8), scale.float().contiguous()


class ServingLayer:
    """Weights, buffers and bound calls of the layer for T tokens a rank."""

    def __init__(self, comm, router, w_router, w_in, w_out, tokens):
        """w_router (E, C); w_in (E, 2 F, C): the gates' rows, then the ups'; w_out (E, C, F)."""
        self.stream = torch.cuda.current_stream()  # which the bound calls keep
        P, E, K = comm.nranks, router.experts, router.top_k
        C, F, dev = w_router.shape[1], w_out.shape[2], w_router.device
        T, each, room = tokens, E // P, P * tokens * K  # (every route of every rank could go to one rank)
        self.comm, self.w_router = comm, w_router
        codes_in, scale_in = quantize_weights(w_in)
        codes_out, scale_out = quantize_weights(w_out)

        def new(*shape, dtype=torch.float32):
            return torch.empty(shape, device=dev, dtype=dtype)

        bf16, i8, i32, i64 = torch.bfloat16, torch.int8, torch.int32, torch.int64
        ranks = range(P)
        self.x = [new(T, C, dtype=bf16) for _ in ranks]
        self.out = [new(T, C, dtype=bf16) for _ in ranks]
        self.logits = [new(T, E) for _ in ranks]
        self.counts, self.back = new(P, P, dtype=i64), new(P, P, dtype=i64)
        self.offsets = new(P, E + 1, dtype=i64)
        self.segments = [torch.zeros(E + 1, device=dev, dtype=i64) for _ in ranks]
        index, weight = [new(T, K, dtype=i32) for _ in ranks], [new(T, K) for _ in ranks]
        row = [new(T, K, dtype=i32) for _ in ranks]
        sent, sent_scale = [new(T * K, C, dtype=i8) for _ in ranks], [new(T * K) for _ in ranks]
        got, got_scale = [new(room, C, dtype=i8) for _ in ranks], [new(room) for _ in ranks]
        hidden, hidden8, hidden_scale = new(room, 2 * F, dtype=bf16), new(room, F, dtype=i8), new(room)
        rows, home = [new(room, C, dtype=bf16) for _ in ranks], [new(T * K, C, dtype=bf16) for _ in ranks]
        space = new(max(1, H.hccl_moe_plan_bytes(T, K, E)), dtype=torch.uint8)

        self.route = [comm.bind_moe_route(router, self.logits[r], index[r], weight[r]) for r in ranks]
        self.plan = [comm.bind_moe_plan(index[r], E, row[r], self.offsets[r], T * K, rank_counts=self.counts[r], workspace=space)
                     for r in ranks]
        self.dispatch = [comm.bind_moe_dispatch(self.x[r], row[r], sent[r], scale=sent_scale[r]) for r in ranks]
        # codes travel as 32-bit elements; the counts that arrive are those of the way back
        self.go = [comm.bind_alltoallv_dynamic([s.view(i32) for s in sent], self.counts, [g.view(i32) for g in got], C // 4,
                                               recvcounts=self.back),
                   comm.bind_alltoallv_dynamic(sent_scale, self.counts, got_scale, 1)]
        self.expert = []
        for r in ranks:
            own, seg = slice(r * each, (r + 1) * each), self.segments[r]
            self.expert += [
                comm.bind_moe_product(got[r], got_scale[r], codes_in[own], scale_in[own], hidden, offsets=seg),
                comm.bind_moe_quantize(hidden, hidden8, hidden_scale, gated=True, limit=seg[-1:]),
                comm.bind_moe_product(hidden8, hidden_scale, codes_out[own], scale_out[own], rows[r], offsets=seg)]
        self.come = comm.bind_alltoallv_dynamic(rows, self.back, home, C)
        self.combine = [comm.bind_moe_combine(home[r], row[r], self.out[r], weight=weight[r]) for r in ranks]

    def __call__(self):
        """self.x (P tensors) -> self.out, in the order of the current stream"""
        here = torch.cuda.current_stream()
        if here == self.stream:
            return self._layer()
        self.stream.wait_stream(here)
        with torch.cuda.stream(self.stream):
            out = self._layer()
        here.wait_stream(self.stream)
        return out

    def _layer(self):
        P = self.comm.nranks
        for r in range(P):
            torch.mm(self.x[r].float(), self.w_router.t(), out=self.logits[r])
            self.route[r]()
            self.plan[r]()
            self.dispatch[r]()
        with self.comm.group():
            for call in self.go:
                call()
        # what a rank received lies source by source, and by expert within a source: segments as they are
        sizes = self.offsets[:, 1:] - self.offsets[:, :-1]
        for r, seg in enumerate(self.segments):
            each = sizes.shape[1] // P
            torch.cumsum(sizes[:, r * each:(r + 1) * each].reshape(-1), 0, out=seg[1:])
        for call in self.expert:
            call()
        self.come()
        for call in self.combine:
            call()
        return self.out


# ---- training --------------------------------------------------------------------------------------

class Route(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, comm, router):
        index = torch.empty(logits.shape[0], router.top_k, device=logits.device, dtype=torch.int32)
        weight = torch.empty(index.shape, device=logits.device)
        comm.moe_route(router, logits, index, weight)
        ctx.save_for_backward(logits, index)
        ctx.comm, ctx.router = comm, router
        ctx.mark_non_differentiable(index)
        return weight, index

    @staticmethod
    def backward(ctx, grad_weight, _):
        logits, index = ctx.saved_tensors
        grad = torch.empty_like(logits)
        ctx.comm.moe_route_backward(ctx.router, logits, index, grad_weight.contiguous(), grad)
        return grad, None, None


class Dispatch(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, row, comm):
        out = x.new_zeros(row.numel(), x.shape[1])
        comm.moe_dispatch(x, row, out)
        ctx.save_for_backward(row)
        ctx.comm = comm
        return out

    @staticmethod
    def backward(ctx, grad):
        (row,) = ctx.saved_tensors
        dx = grad.new_empty(row.shape[0], grad.shape[1])
        ctx.comm.moe_combine(grad.contiguous(), row, dx)
        return dx, None, None


class Combine(torch.autograd.Function):
    @staticmethod
    def forward(ctx, z, weight, row, comm):
        out = z.new_empty(row.shape[0], z.shape[1])
        comm.moe_combine(z, row, out, weight=weight)
        ctx.save_for_backward(z, weight, row)
        ctx.comm = comm
        return out

    @staticmethod
    def backward(ctx, grad):
        z, weight, row = ctx.saved_tensors
        dz, dw = torch.zeros_like(z), torch.empty_like(weight)
        ctx.comm.moe_combine_backward(grad.contiguous(), z, row, weight, dz, dw)
        return dz, dw, None, None


def expert_rows(x, offsets, w_in, w_out):
    """The experts on rows in their order, each by plain products (the sizes are read on the host)."""
    out, F = [], w_out.shape[2]
    for e, (a, b) in enumerate(zip(offsets[:-1], offsets[1:])):
        h = x[a:b] @ w_in[e].t()
        out.append((torch.nn.functional.silu(h[:, :F]) * h[:, F:]) @ w_out[e].t())
    return torch.cat(out + [x[offsets[-1]:] * 0])


def train_step(comm, router, x, w_router, w_in, w_out):
    """The layer's result; its gradients by .backward()."""
    logits = x @ w_router.t()
    weight, index = Route.apply(logits, comm, router)
    row = torch.empty_like(index)
    offsets = torch.empty(router.experts + 1, device=x.device, dtype=torch.int64)
    space = torch.empty(max(1, H.hccl_moe_plan_bytes(*index.shape, router.experts)), device=x.device, dtype=torch.uint8)
    comm.moe_plan(index, router.experts, row, offsets, index.numel(), workspace=space)
    rows = Dispatch.apply(x, row, comm)
    return Combine.apply(expert_rows(rows, offsets.tolist(), w_in, w_out), weight, row, comm)


# ---- both, checked ---------------------------------------------------------------------------------

def plain_layer(x, router, w_router, w_in, w_out):
    """The layer in 32 bits, every token through its experts."""
    x, F = x.float(), w_out.shape[2]
    p = torch.softmax(x @ w_router.float().t(), 1)
    top, index = p.topk(router.top_k, 1)
    weight = top / top.sum(1, keepdim=True) * router.scale
    y = torch.zeros_like(x)
    for e in range(router.experts):
        h = x @ w_in[e].float().t()
        z = (torch.nn.functional.silu(h[:, :F]) * h[:, F:]) @ w_out[e].float().t()
        y = y + (weight * (index == e)).sum(1, keepdim=True) * z
    return y


def parameters(seed, E, C, F, dtype, device="cuda:0"):
    g = torch.Generator(device=device)
    g.manual_seed(seed)

    def normal(*shape):
        return (torch.randn(shape, generator=g, device=device) * shape[-1] ** -0.5).to(dtype)

    return normal(E, C), normal(E, 2 * F, C), normal(E, C, F)


def serve(ranks=8, tokens=48, experts=32, top_k=4, hidden=512, inner=256):
    """The relative error of the 8-bit layer against the layer in 32 bits."""
    router = H.hccl_router_init(experts=experts, top_k=top_k, renormalize=True)
    w_router, w_in, w_out = parameters(0, experts, hidden, inner, torch.float32)
    with H.Comm(ranks, device=0) as comm:
        layer = ServingLayer(comm, router, w_router, w_in, w_out, tokens)
        worst = 0.0
        for step in range(3):
            g = torch.Generator(device="cuda:0")
            g.manual_seed(10 + step)
            for r in range(ranks):
                layer.x[r].copy_(torch.randn(tokens, hidden, generator=g, device="cuda:0"))
            out = layer()
            for r in range(ranks):
                want = plain_layer(layer.x[r], router, w_router, w_in, w_out)
                worst = max(worst, float((out[r].float() - want).norm() / want.norm()))
        if comm.async_error() != 0:
            raise RuntimeError(H.hccl_get_last_error())
    return worst


def train(tokens=200, experts=16, top_k=2, hidden=64, inner=32):
    """The greatest error of the result and of every gradient against the plain layer's, of their size, or
    of 1 where that is less: the router of one choice, renormalised, has weight 1 and no gradient."""
    router = H.hccl_router_init(experts=experts, top_k=top_k, renormalize=True)
    weights = parameters(1, experts, hidden, inner, torch.float32)
    g = torch.Generator(device="cuda:0")
    g.manual_seed(2)
    x, dy = (torch.randn(tokens, hidden, generator=g, device="cuda:0") for _ in range(2))
    results = []
    with H.Comm(1, device=0) as comm:
        for layer in (lambda *a: train_step(comm, router, *a), lambda *a: plain_layer(a[0], router, *a[1:])):
            inputs = [t.clone().requires_grad_() for t in (x, *weights)]
            y = layer(*inputs)
            y.backward(dy)
            results.append([y.detach()] + [t.grad for t in inputs])
    return max(float((a - b).norm() / b.norm().clamp(min=1.0)) for a, b in zip(*results))


if __name__ == "__main__":
    print(f"serving, 8-bit experts: relative error {serve():.4f} against the layer in 32 bits")
    print(f"training, result and gradients: relative error {train():.2e}")
