"""The example: a layer of experts trained and served with the library's
16-bit products."""
import os
import subprocess
import sys

import pytest

import gpu_util

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.join(ROOT, "examples"))


@pytest.fixture(scope="module", autouse=True)
def gpu():
    gpu_util.require_gpu()


def test_training_lowers_the_loss():
    import expert_layer
    losses = expert_layer.train(tokens=1024, width=128, inner=256, experts=4, steps=30, say=None)
    assert all(x == x for x in losses) and losses[-1] < 0.8 * losses[0], losses


def test_gradients_are_those_of_the_layer():
    """The layer's gradients against the same layer written with torch's own
    products, in 32 bits on the same 16-bit weights: within bfloat16's
    rounding of the activations (a few 2^-8 in the 2-norm)."""
    import torch
    import torch.nn.functional as F
    import expert_layer
    gen = torch.Generator(device="cuda").manual_seed(0)
    n = lambda *s: torch.randn(s, device="cuda", generator=gen)  # noqa: E731
    X, router = n(300, 64).bfloat16(), (n(64, 4) / 8).bfloat16()
    up, down = (n(4, 96, 64) / 8).bfloat16().requires_grad_(), (n(4, 64, 96) / 10).bfloat16().requires_grad_()
    dY = n(300, 64).bfloat16()
    expert_layer.expert_layer(X, router, up, down).backward(dY)
    up32, down32 = (w.detach().float().requires_grad_() for w in (up, down))
    gate, which = torch.softmax((X @ router).float(), -1).topk(2)
    Y = torch.zeros(300, 64, device="cuda")
    for e in range(4):
        for c in range(2):
            at = torch.nonzero(which[:, c] == e).flatten()
            h = F.silu(X[at].float() @ up32[e].t())
            Y = Y.index_add(0, at, (h @ down32[e].t()) * gate[at, c, None])
    Y.backward(dY.float())
    for got, want in ((up.grad, up32.grad), (down.grad, down32.grad)):
        assert float((got.float() - want).norm() / want.norm()) < 4 * 2.0 ** -8


def test_served_requests():
    import expert_layer
    assert expert_layer.serve(requests=40, say=None) < 2.0 ** -7


def test_command():
    out = subprocess.run([sys.executable, os.path.join(ROOT, "examples", "expert_layer.py"), "--tokens", "512",
                          "--width", "64", "--inner", "128", "--experts", "4", "--steps", "2"], capture_output=True,
                         text=True, timeout=110)
    assert out.returncode == 0, out.stderr[-2000:]
    assert "loss" in out.stdout and "served" in out.stdout
