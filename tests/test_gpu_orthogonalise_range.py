"""The orthogonalisation at the ends of its arguments' ranges: matrices of
zeros, inputs at either end of float32's range, polynomials whose values grow
past what half holds, on the path of one launch (at most 128 x 128) and on the
path of tiles."""
import pytest
import torch

import gpu_util
import paper_2609_09095_amd as oz
from test_gpu_orthogonalise import MUON, exact, gradient

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


def rank_one(shape):
    gen = torch.Generator(device="cuda").manual_seed(1)
    n = lambda *s: torch.randn(s, device="cuda", generator=gen)  # noqa: E731
    return n(*shape[:-1], 1) * n(*shape[:-2], 1, shape[-1])


def rounded(x):
    """To half's 11 bits at any exponent."""
    m, e = torch.frexp(x)
    return torch.ldexp(torch.round(m * 2048) / 2048, e)


@pytest.mark.parametrize("coefficients, steps", [
    ((7.9, 0.0, 0.0), 2),       # singular values of 7.9 before the last step
    ((2.0, 250.0, 0.0), 1), ((-2.0, 0.0, -250.0), 1),  # |b s^2 + c s^4| of 250
    ((2.0, 1.5, 0.5), 2), ((3.0, -4.0, 2.0), 6), ((-7.0, 3.0, 0.0), 2), ((1e-3, 0.0, 0.0), 3), (MUON, 5)])
@pytest.mark.parametrize("shape", SHAPES)
def test_polynomials_inside_the_stated_range(shape, coefficients, steps):
    """Matrices of rank one, whose singular value is 1 at first: with operands
    of 11 bits the results are as near as the model with such operands is,
    twice, beside the result's rounding."""
    G = rank_one(shape)
    X = call(G, coefficients=coefficients, steps=steps)
    for x, g in zip(X, G):
        want = exact(g, steps, coefficients)
        d = (exact(g, steps, coefficients, operand=rounded) - want).norm()
        off = (x.double() - want).norm()
        assert off <= 2 * d + (2.0 ** -9 + 1e-5) * want.norm(), (float(off / want.norm()), float(d / want.norm()))


@pytest.mark.parametrize("coefficients, steps", [((1e4, 0.0, 0.0), 3), ((2.0, 1e5, 0.0), 2), ((0.0, 0.0, 1e6), 3)])
@pytest.mark.parametrize("shape", SHAPES)
def test_polynomials_past_the_stated_range_do_not_pass_for_results(shape, coefficients, steps):
    assert not torch.isfinite(call(rank_one(shape), coefficients=coefficients, steps=steps)).any()
