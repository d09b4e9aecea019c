"""Matrices of few directions (gradients of few tokens): every rounding that
leaves those directions is noise that later steps multiply by a.  The
tolerance is the one of the full matrices' tests."""
import pytest
import torch

import gpu_util
from test_gpu_orthogonalise import check

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def gpu():
    gpu_util.require_gpu()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rank", [1, 4, 16, 32, 64])
@pytest.mark.parametrize("shape", [(2, 96, 128), (2, 128, 40), (2, 64, 64), (2, 264, 130), (1, 300, 520), (1, 1000, 1000)])
def test_few_directions(shape, rank, dtype):
    gen = torch.Generator(device="cuda").manual_seed(rank)
    n = lambda *s: torch.randn(s, device="cuda", generator=gen)  # noqa: E731
    check((n(*shape[:-1], rank) @ n(*shape[:-2], rank, shape[-1])).to(dtype))


@pytest.mark.parametrize("steps", [1, 2, 5, 8])
@pytest.mark.parametrize("shape", [(3, 2, 9), (2, 102, 2), (7, 4, 12), (3, 8, 8), (3, 7, 1200), (2, 16, 113), (3, 192, 32), (2, 64, 448)])
def test_few_rows_of_few_directions(shape, steps):
    gen = torch.Generator(device="cuda").manual_seed(sum(shape))
    n = lambda *s: torch.randn(s, device="cuda", generator=gen)  # noqa: E731
    for rank in (1, 2, 3, 5, 12, 24):
        if rank < min(shape[1:]):
            check(n(*shape[:-1], rank) @ n(*shape[:-2], rank, shape[-1]), steps=steps)


@pytest.mark.parametrize("shape", [(1, 96, 128), (1, 130, 264), (1, 1000, 700)])
def test_singular_values_over_three_decades(shape):
    gen = torch.Generator(device="cuda").manual_seed(5)
    U, s, V = torch.linalg.svd(torch.randn(shape, dtype=torch.float64, device="cuda", generator=gen), full_matrices=False)
    s = torch.logspace(0, -3, s.shape[-1], dtype=torch.float64, device="cuda")
    check((U * s @ V).float())
    check((U * s @ V).float(), coefficients=(1.5, -0.5, 0.0), steps=12)


@pytest.mark.parametrize("shape", [(2, 96, 128), (1, 300, 520)])
def test_no_fifth_power(shape):
    gen = torch.Generator(device="cuda").manual_seed(9)
    n = lambda *s: torch.randn(s, device="cuda", generator=gen)  # noqa: E731
    for G in (n(*shape), n(*shape[:-1], 8) @ n(*shape[:-2], 8, shape[-1])):
        check(G, coefficients=(1.5, -0.5, 0.0), steps=8)
