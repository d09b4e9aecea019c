"""The orthogonalisation at the ends of its arguments' ranges: matrices of
zeros, inputs at either end of float32's range, polynomials whose values grow
past what half holds, on the path of one launch (at most 128 x 128) and on the
path of tiles."""
import pytest
import torch

import gpu_util
import paper_2609_09095_amd as oz
from test_gpu_orthogonalise import gradient

pytestmark = pytest.mark.gpu

SHAPES = [(2, 96, 128), (2, 128, 40), (1, 300, 520), (2, 264, 130)]


@pytest.fixture(scope="module", autouse=True)
def gpu():
    gpu_util.require_gpu()


def call(G, **kw):
    gpu_util.log(f"orthogonalise {tuple(G.shape)} {G.dtype} {kw}")
    X = oz.ozaki25_orthogonalise(G, **kw)
    torch.cuda.synchronize()
    return X


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("shape", SHAPES)
def test_zeros_stay_zeros(shape, dtype):
    """Also where eps, or its reciprocal in 32 bits, gives no finite scale."""
    for eps in (0.0, 1e-42, 1e-7):
        assert torch.count_nonzero(call(torch.zeros(shape, dtype=dtype, device="cuda"), eps=eps)) == 0
        G = gradient(shape, dtype)
        G[0] = 0
        X = call(G, eps=eps)
        assert torch.count_nonzero(X[0]) == 0 and torch.isfinite(X).all()


@pytest.mark.parametrize("exponent", [-149, -140, -120, 0, 100, 118])
@pytest.mark.parametrize("shape", SHAPES)
def test_norms_whose_reciprocal_is_no_normal_float(shape, exponent):
    """Whole numbers up to 2^9 times a power of two, the least one float32's
    least positive number: scaling is exact, so results are equal."""
    G = (gradient(shape, torch.float32) * 6e4).round().clamp(-511, 511)
    assert float(G.abs().max()) > 100
    assert torch.equal(call(G, eps=0.0), call(torch.ldexp(G.double(), torch.tensor(exponent, device="cuda")).float(), eps=0.0))
