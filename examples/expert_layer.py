"""A layer of experts, trained and served.

    python examples/expert_layer.py [--tokens 4096] [--width 512] [--inner 1024] [--experts 8] [--steps 20]

Training: tokens are routed to two experts each, sorted by expert and sent
through the experts' two projections; the backward pass gives the inputs' and
the weights' gradients; the update is the momentum orthogonalised per expert.
Serving: a batch of requests, each with a low-rank adapter of its own, goes
through a projection that they share, one token per request.

Every product with weights is one of the library's calls; the rest is torch.
"""
import argparse
import os
import sys

import torch
import torch.nn.functional as F

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import paper_2609_09095_amd as oz  # noqa: E402


class GroupedLinear(torch.autograd.Function):
    """Y[r] = X[r] W[g]^T for rows sorted by group; dW in 32 bits."""

    @staticmethod
    def forward(ctx, X, W, ends):
        ctx.save_for_backward(X, W, ends)
        return oz.ozaki25_grouped_matmul(X, W, ends)

    @staticmethod
    def backward(ctx, dY):
        X, W, ends = ctx.saved_tensors
        dY = dY.contiguous()
        dX = oz.ozaki25_grouped_matmul_dx(dY, W, ends)
        dW = oz.ozaki25_grouped_matmul_dw(dY, X, ends, out_dtype=torch.float32)
        return dX, dW.to(W.dtype), None


def expert_layer(X, router, up, down, top=2):
    """X: tokens x width.  Every token's sum over its `top` experts, weighted
    by the router."""
    gate, which = torch.softmax((X @ router).float(), -1).topk(top)
    order = which.flatten().argsort(stable=True)  # rows (token, choice) by expert
    ends = torch.bincount(which.flatten(), minlength=up.shape[0]).cumsum(0).to(torch.int32)
    rows = X[order // top]
    hidden = F.silu(GroupedLinear.apply(rows, up, ends))
    out = GroupedLinear.apply(hidden, down, ends) * gate.flatten()[order, None].to(X.dtype)
    return torch.zeros_like(X).index_add(0, order // top, out)


def train(tokens=4096, width=512, inner=1024, experts=8, steps=20, rate=0.02, decay=0.95, seed=0, say=print):
    """Fits the layer to a fixed random map; returns the losses."""
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, scale=1.0):
        return (torch.randn(shape, device="cuda", generator=gen) * scale).to(torch.bfloat16)

    router = normal(width, experts, scale=width ** -0.5)
    masters = [torch.randn(s, device="cuda", generator=gen) * s[2] ** -0.5
               for s in ((experts, inner, width), (experts, width, inner))]
    momenta = [torch.zeros_like(w) for w in masters]
    rooms = [torch.empty(oz.ozaki25_orthogonalise_workspace_size(*w.shape), dtype=torch.uint8, device="cuda")
             for w in masters]
    target = normal(width, width, scale=width ** -0.5)
    losses = []
    for step in range(steps):
        X = normal(tokens, width)
        weights = [w.to(torch.bfloat16).requires_grad_() for w in masters]
        Y = expert_layer(X, router, *weights)
        loss = (Y.float() - (X @ target).float()).square().mean()
        loss.backward()
        for master, momentum, room, w in zip(masters, momenta, rooms, weights):
            momentum.mul_(decay).add_(w.grad.float())
            update = oz.ozaki25_orthogonalise(momentum, workspace=room)
            n, k = master.shape[1:]
            master.add_(update.float(), alpha=-rate * max(1.0, n / k) ** 0.5)
        losses.append(float(loss.detach()))
        if say and (step % 5 == 0 or step + 1 == steps):
            say(f"step {step:3d}  loss {losses[-1]:.4f}")
    return losses


def serve(requests=32, width=512, adapters=16, rank=16, seed=1, say=print):
    """One token of each request through the shared projection and the
    request's own adapter; returns the largest difference from a request at a
    time in 32 bits, relative to the outputs."""
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, scale=1.0):
        return (torch.randn(shape, device="cuda", generator=gen) * scale).to(torch.bfloat16)

    X, W = normal(requests, width), normal(width, width, scale=width ** -0.5)
    A, B = normal(adapters, rank, width, scale=width ** -0.5), normal(adapters, width, rank, scale=0.25)
    ids = torch.randint(-1, adapters, (requests,), device="cuda", generator=gen, dtype=torch.int32)
    scales = torch.full((adapters,), 0.5, device="cuda")
    Y = oz.ozaki25_adapter_matmul(X, W, ids, A, B, scales)
    worst = 0.0
    for t, a in enumerate(ids.tolist()):
        y = X[t].float() @ W.float().t()
        if a >= 0:
            y += 0.5 * (B[a].float() @ (A[a].float() @ X[t].float()))
        worst = max(worst, float((Y[t].float() - y).abs().max() / y.abs().max()))
    if say:
        say(f"served {requests} requests with {adapters} adapters: largest difference {worst:.1e}")
    return worst


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("tokens", 4096), ("width", 512), ("inner", 1024), ("experts", 8), ("steps", 20)):
        ap.add_argument(f"--{name}", type=int, default=value)
    a = ap.parse_args()
    train(a.tokens, a.width, a.inner, a.experts, a.steps)
    serve(width=a.width)


if __name__ == "__main__":
    main()
