"""A projection trained in 8 bits behind its norm, and a decode step through a layer
of experts whose weights are in 8 bits.

    python examples/eight_bit_block.py [--rows 512] [--width 256] [--out 384] [--steps 10]

Training: the residual is added, the norm writes the product's operand in 8 bits, and
the three products (output, input's gradient, weights' gradient) run on e4m3 numbers
with a scale per block of 128.  Serving: one token of each request through the norm, a
projection and the experts that its router chose.

Every product, norm and quantisation is one of the library's calls; the rest is torch.
"""
import argparse
import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import paper_2609_09095_amd as oz  # noqa: E402


class NormLinear(torch.autograd.Function):
    """H = X + residual, Y = norm(H) W^T: returns (Y, H).  W: out x width in 32 bits,
    quantised in squares; its gradient in 32 bits."""

    @staticmethod
    def forward(ctx, X, residual, weight, W, eps):
        Q, scales, H = oz.ozaki25_rms_norm(X, weight, residual=residual, eps=eps, quantised=True)
        w, ws, wt, wts = oz.ozaki25_quantise(W, squares=True, layout="both")
        ctx.save_for_backward(H, weight, wt, wts)
        ctx.eps = eps
        return oz.ozaki25_scaled_matmul(Q, scales, w, ws, out_dtype=X.dtype), H

    @staticmethod
    def backward(ctx, dY, dH):
        H, weight, wt, wts = ctx.saved_tensors
        with torch.no_grad():
            y, ys, yt, yts = oz.ozaki25_quantise(dY.contiguous(), layout="both")
            dN = oz.ozaki25_scaled_matmul(y, ys, wt, wts, out_dtype=H.dtype)
            # the norm again, with scales along the rows: the operand of the weights' gradient
            N = oz.ozaki25_rms_norm(H, weight, eps=ctx.eps)
            nt, nts = oz.ozaki25_quantise(N, layout="columns")
            dW = oz.ozaki25_scaled_matmul(yt, yts, nt, nts, squares=False, out_dtype=torch.float32)
            dX, dweight = oz.ozaki25_rms_norm_backward(dN, H, weight, dH=dH.contiguous(), eps=ctx.eps)
        return dX, dX, dweight.to(weight.dtype), dW, None


def train(rows=512, width=256, out=384, steps=10, rate=0.05, seed=0, say=print):
    """Fits the projection to a fixed random map; returns the losses."""
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, scale=1.0):
        return torch.randn(shape, device="cuda", generator=gen) * scale

    W = normal(out, width, scale=width ** -0.5).requires_grad_()
    weight = torch.ones(width, device="cuda", dtype=torch.bfloat16).requires_grad_()
    target = normal(width, out, scale=width ** -0.5)
    losses = []
    for step in range(steps):
        X, residual = normal(rows, width).bfloat16(), normal(rows, width).bfloat16()
        Y, H = NormLinear.apply(X, residual, weight, W, 1e-6)
        h = H.float()
        want = (h / h.square().mean(1, keepdim=True).sqrt()) @ target
        loss = (Y.float() - want).square().mean()
        loss.backward()
        with torch.no_grad():
            W -= rate * W.grad * rows
            W.grad = weight.grad = None
        losses.append(float(loss.detach()))
        if say:
            say(f"step {step:3d}  loss {losses[-1]:.4f}")
    return losses


class Decoder:
    """The weights of a block's second half as a server keeps them, and its decode step."""

    def __init__(self, width=256, inner=128, experts=8, top=2, seed=1):
        gen = torch.Generator(device="cuda").manual_seed(seed)

        def normal(*shape):
            return torch.randn(shape, device="cuda", generator=gen) * shape[-1] ** -0.5

        self.top, self.eps = top, 1e-6
        self.norms = [(1 + 0.1 * torch.randn(width, device="cuda", generator=gen)).bfloat16() for _ in range(2)]
        self.proj, self.proj_scales = oz.ozaki25_quantise(normal(width, width), squares=True)
        self.router = normal(experts, width).bfloat16()
        self.up, self.up_scales = oz.ozaki25_quantise(normal(experts, inner, width), squares=True)
        self.gate, self.gate_scales = oz.ozaki25_quantise(normal(experts, inner, width), squares=True)
        self.down, self.down_scales = oz.ozaki25_quantise(normal(experts, width, inner), squares=True)

    def room(self, tokens):
        inner, width = self.up.shape[1:]
        return torch.empty((oz.ozaki25_expert_layer_workspace_size(tokens, self.top, width, inner, width),), dtype=torch.uint8,
                           device="cuda")

    def step(self, X, residual, room=None):
        """X: tokens x width, what the block before added; returns (X, residual) for the
        block after, and what was computed on the way."""
        Q, scales, H = oz.ozaki25_rms_norm(X, self.norms[0], residual=residual, eps=self.eps, quantised=True)
        P = oz.ozaki25_scaled_matmul(Q, scales, self.proj, self.proj_scales)
        N, H2 = oz.ozaki25_rms_norm(P, self.norms[1], residual=H, eps=self.eps)
        gates, which = torch.softmax((N @ self.router.t()).float(), -1).topk(self.top)
        gates, which = gates / gates.sum(-1, keepdim=True), which.to(torch.int32)
        Y = oz.ozaki25_expert_layer(N, which, gates, self.up, self.down, gate=self.gate, up_scales=self.up_scales,
                                    down_scales=self.down_scales, gate_scales=self.gate_scales, workspace=room)
        return Y, H2, {"Q": Q, "scales": scales, "H": H, "P": P, "N": N, "which": which, "gates": gates}


def serve(requests=16, width=256, seed=1, say=print):
    """A decode step of as many requests, captured once and replayed for new tokens;
    returns the largest difference between the replay and the same step run alone."""
    block = Decoder(width=width, seed=seed)
    gen = torch.Generator(device="cuda").manual_seed(seed + 1)
    X, residual = (torch.zeros((requests, width), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    room = block.room(requests)
    block.step(X, residual, room)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        Y, H, _ = block.step(X, residual, room)
    worst = 0.0
    for _ in range(3):
        for t in (X, residual):
            t.copy_(torch.randn((requests, width), device="cuda", generator=gen))
        graph.replay()
        torch.cuda.synchronize()
        y, h, _ = block.step(X, residual)
        worst = max(worst, float((Y.float() - y.float()).abs().max()), float((H.float() - h.float()).abs().max()))
    if say:
        say(f"served {requests} requests, three tokens each: largest difference {worst:.1e}")
    return worst


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("rows", 512), ("width", 256), ("out", 384), ("steps", 10)):
        ap.add_argument(f"--{name}", type=int, default=value)
    a = ap.parse_args()
    train(a.rows, a.width, a.out, a.steps)
    serve(width=a.width)


if __name__ == "__main__":
    main()
