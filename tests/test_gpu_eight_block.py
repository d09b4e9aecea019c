"""The 8-bit path's operators together, as a block uses them: a decode step link by
link, a projection's training step, captured graphs, other streams, the example."""
import os
import subprocess
import sys

import pytest

import gpu_util
import paper_2609_09095_amd as oz

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.join(ROOT, "examples"))


@pytest.fixture(scope="module", autouse=True)
def gpu():
    gpu_util.require_gpu()


@pytest.mark.parametrize("requests", [1, 7, 33])
def test_decode_step_link_by_link(requests):
    """Each link's output against the formula on what the link before it gave."""
    import torch
    import eight_bit_block
    import eight_util as u
    import test_gpu_layer as layer
    import test_gpu_norm as norm
    width, inner = 200, 100
    block = eight_bit_block.Decoder(width=width, inner=inner)
    X, R = u.normal((requests, width), torch.bfloat16, 3), u.normal((requests, width), torch.bfloat16, 4)
    Y, H2, way = block.step(X, R, block.room(requests))
    H, want = norm.expected(X, R, block.norms[0])
    assert torch.equal(way["H"], H)
    s = u.spread(way["scales"], requests, width).double()
    u.assert_e4m3(way["Q"], want / s, 38 * u.U)
    W = block.proj.double() * u.spread(block.proj_scales, width, width, True).double()
    P = (way["Q"].double() * s) @ W.t()
    size = (way["Q"].double() * s).abs() @ W.abs().t()
    assert bool(((way["P"].double() - P).abs() <= P.abs() * 2.0 ** -8 + size * 2.0 ** -10).all())
    H, want = norm.expected(way["P"], way["H"], block.norms[1])
    assert torch.equal(H2, H)
    norm.close(way["N"], want, X.dtype, 35 * u.U)
    V = [torch.stack([q.double() * u.spread(c, *q.shape, True).double() for q, c in zip(Q, sc)])
         for Q, sc in ((block.up, block.up_scales), (block.gate, block.gate_scales), (block.down, block.down_scales))]
    want, off = layer.expected(way["N"], way["which"], way["gates"], V[0], V[1], V[2])
    assert bool(((Y.double() - want).abs() <= off + (want.abs() + off) * 2.0 ** -8).all())


def test_training_step():
    """The gradients that the example's projection gives against those of the same
    function in 64 bits.  Each operand of a product is rounded to e4m3 once (2^-4 of a
    number at most, so of a product's 2-norm 2^-4 for each operand, as the roundings do
    not depend on each other's place), the norm's operand feeds both."""
    import torch
    import eight_bit_block
    import eight_util as u
    rows, width, out = 300, 200, 150
    X, R = u.normal((rows, width), torch.bfloat16, 1).requires_grad_(), u.normal((rows, width), torch.bfloat16, 2).requires_grad_()
    weight = (1 + 0.2 * u.normal((width,), torch.float32, 3)).bfloat16().requires_grad_()
    W = u.normal((out, width), torch.float32, 4, width ** -0.5).requires_grad_()
    dY, dH = u.normal((rows, out), torch.bfloat16, 5), u.normal((rows, width), torch.bfloat16, 6)
    Y, H = eight_bit_block.NormLinear.apply(X, R, weight, W, 1e-6)
    torch.autograd.backward([Y, H], [dY, dH])
    h = (X.detach().float() + R.detach().float()).bfloat16().double().requires_grad_()
    v, w = weight.detach().double().requires_grad_(), W.detach().double().requires_grad_()
    y = (h / (h.square().mean(1, keepdim=True) + 1e-6).sqrt() * v) @ w.t()
    torch.autograd.backward([y, h], [dY.double(), dH.double()])
    assert torch.equal(H.double(), h.detach()) and torch.equal(X.grad, R.grad)
    for got, want in ((Y, y), (X.grad, h.grad), (W.grad, w.grad), (weight.grad, v.grad)):
        got, want = got.detach().double(), want.detach()
        assert float((got - want).norm() / want.norm()) < 2 * 2.0 ** -4


def calls():
    """name -> (inputs, call): one of every entry point, with a workspace where it takes
    one, the inputs in place."""
    import torch
    import eight_util as u
    room = lambda n: torch.empty(max(n, 1), dtype=torch.uint8, device="cuda")  # noqa: E731
    found = {}
    X, R, w = u.normal((70, 300), torch.bfloat16, 1), u.normal((70, 300), torch.bfloat16, 2), u.normal((300,), torch.bfloat16, 3)
    found["norm"] = ([X, R, w], lambda X=X, R=R, w=w: oz.ozaki25_rms_norm(X, w, residual=R, quantised=True))
    a, b, c = (t.clone() for t in (X, R, w))
    back = room(oz.ozaki25_rms_norm_backward_workspace_size(70, 300))
    found["norm_backward"] = ([a, b, c], lambda: oz.ozaki25_rms_norm_backward(a, b, c, workspace=back))
    q = u.normal((3, 150, 140), torch.float32, 4)
    found["quantise"] = ([q], lambda: oz.ozaki25_quantise(q, layout="both"))
    for name, (rows, n, k) in {"few": (5, 200, 600), "tiles": (300, 200, 600), "parts": (100, 70, 6200), "many": (2100, 2050, 300)}.items():
        x, y = u.normal((rows, k), torch.float32, 5), u.normal((n, k), torch.float32, 6)
        A, s = oz.ozaki25_quantise(x)
        B, t = oz.ozaki25_quantise(y, squares=True)
        space = room(oz.ozaki25_scaled_matmul_workspace_size(rows, n, k))
        found["matmul_" + name] = ([A.view(torch.uint8), s], lambda A=A, s=s, B=B, t=t, space=space: oz.ozaki25_scaled_matmul(
            A, s, B, t, workspace=space))
    for tokens in (2, 40):
        h = u.normal((tokens, 256), torch.bfloat16, 7)
        up, down = u.normal((6, 100, 256), torch.bfloat16, 8, 1 / 16), u.normal((6, 256, 100), torch.bfloat16, 9, 0.1)
        which = torch.randint(-1, 6, (tokens, 3), device="cuda", dtype=torch.int32)
        gates = torch.rand((tokens, 3), device="cuda")
        space = room(oz.ozaki25_expert_layer_workspace_size(tokens, 3, 256, 100, 256))
        found[f"layer_{tokens}"] = ([h, which, gates], lambda h=h, which=which, gates=gates, up=up, down=down, space=space:
                                    oz.ozaki25_expert_layer(h, which, gates, up, down, gate=up, workspace=space))
    return found


NAMES = ["norm", "norm_backward", "quantise", "matmul_few", "matmul_tiles", "matmul_parts", "matmul_many", "layer_2", "layer_40"]


def same(a, b):
    import torch
    a, b = (x if isinstance(x, tuple) else (x,) for x in (a, b))
    return all(torch.equal(x.contiguous().view(torch.uint8), y.contiguous().view(torch.uint8)) for x, y in zip(a, b))


def renew(inputs, seed):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(seed)
    for t in inputs:
        if t.dtype == torch.int32:
            t.copy_(torch.randint(-1, 6, t.shape, device="cuda", generator=gen))
        elif t.dtype == torch.uint8:
            v = torch.randint(0, 126, t.shape, device="cuda", generator=gen) + 128 * torch.randint(0, 2, t.shape, device="cuda", generator=gen)
            t.copy_(v)
        else:
            t.copy_(torch.randn(t.shape, device="cuda", generator=gen).abs() + 0.1 if t.dim() == 1 else
                    torch.randn(t.shape, device="cuda", generator=gen))


@pytest.mark.parametrize("name", NAMES)
def test_captured_and_replayed(name):
    """Replays with new inputs, eager calls and synchronisations between them, against
    the eager results; a second graph over the same workspace runs after the first."""
    import torch
    inputs, call = calls()[name]
    call()
    torch.cuda.synchronize()
    graphs, outs = [], []
    for _ in range(2):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            outs.append(call())
    for seed in range(4):
        renew(inputs, seed)
        for graph, out in zip(graphs, outs):
            graph.replay()
            torch.cuda.synchronize()
            assert same(out, call())
        graphs[0].replay()
        graphs[1].replay()
        torch.cuda.synchronize()
        assert same(outs[0], outs[1])


@pytest.mark.parametrize("name", NAMES)
def test_on_another_stream(name):
    """The current stream of the caller's, twice at once with other inputs in between."""
    import torch
    inputs, call = calls()[name]
    want = call()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = call()
    side.synchronize()
    assert same(got, want)


@pytest.mark.parametrize("name", ["norm", "quantise", "matmul_tiles", "layer_2"])
def test_stream_argument(name):
    import torch
    import eight_util as u
    side = torch.cuda.Stream()
    X = u.normal((40, 256), torch.bfloat16, 1)
    torch.cuda.synchronize()
    if name == "norm":
        call = lambda **kw: oz.ozaki25_rms_norm(X, None, residual=X, **kw)  # noqa: E731
    elif name == "quantise":
        call = lambda **kw: oz.ozaki25_quantise(X, **kw)  # noqa: E731
    elif name == "matmul_tiles":
        Q, s = oz.ozaki25_quantise(X)
        call = lambda **kw: oz.ozaki25_scaled_matmul(Q, s, Q, s, squares=False, **kw)  # noqa: E731
    else:
        which, gates = torch.zeros((40, 1), dtype=torch.int32, device="cuda"), torch.ones((40, 1), device="cuda")
        up = u.normal((2, 64, 256), torch.bfloat16, 2)
        down = u.normal((2, 256, 64), torch.bfloat16, 2)
        call = lambda **kw: oz.ozaki25_expert_layer(X, which, gates, up, down, **kw)  # noqa: E731
    want = call()
    torch.cuda.synchronize()
    for stream in (side, side.cuda_stream):
        got = call(stream=stream)
        side.synchronize()
        assert same(got, want)


def test_example_runs():
    import eight_bit_block
    losses = eight_bit_block.train(rows=256, width=128, out=100, steps=3, say=None)
    assert all(x == x and x < float("inf") for x in losses)
    assert eight_bit_block.serve(requests=5, width=128, say=None) == 0.0


def test_example_command():
    out = subprocess.run([sys.executable, os.path.join(ROOT, "examples", "eight_bit_block.py"), "--rows", "128", "--width", "64",
                          "--out", "96", "--steps", "2"], capture_output=True, text=True, timeout=110)
    assert out.returncode == 0, out.stderr[-2000:]
    assert "loss" in out.stdout and "served" in out.stdout
