"""The model of the orthogonalisation's roundings is fine enough to tell
diagonals kept in 32 bits from rounded ones (on the CPU; the GPU's results are
held to it in test_gpu_orthogonalise_model.py)."""
import pytest
import torch

from orth_model import bound, model
from test_gpu_orthogonalise import exact


@pytest.mark.parametrize("shape", [(300, 520), (515, 300), (128, 128), (96, 128), (128, 64)])
def test_rounded_diagonals_are_told_apart(shape):
    scale = 32.0 if max(shape) <= 128 else 256.0
    torch.manual_seed(0)
    G = torch.randn(shape) + 0.5 * torch.randn(shape[0], 1) * torch.randn(1, shape[1])
    want, right = model(G, scale_x=scale), exact(G)
    planted = model(G, scale_x=scale, diagonals_apart=False).bfloat16().double()
    assert (want.bfloat16().double() - want).norm() <= bound(want, right)
    assert (planted - want).norm() > 1.1 * bound(want, right), ((planted - want).norm() / bound(want, right),)
