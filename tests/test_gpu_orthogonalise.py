"""The Newton-Schulz orthogonalisation against the same steps in 64 bits.

Tolerance: the header says where the operator rounds -- the operands X, S and P
of its products to half, everything else in at least 32 bits, the result to
bfloat16.  `model` takes those roundings in 64-bit arithmetic; its distance d
from the exact steps (2-norm over a matrix) is what they cost.  The kernel may
be 2 d away, plus the rounding of the result (2^-9 of each value, half the
spacing) and 1e-5 of the result for the FP32 sums.
"""
import pytest
import torch

import gpu_util
import paper_2609_09095_amd as oz

pytestmark = pytest.mark.gpu

MUON = (3.4445, -4.7750, 2.0315)


@pytest.fixture(scope="module", autouse=True)
def gpu():
    gpu_util.require_gpu()


def exact(G, steps=5, coefficients=MUON, eps=1e-7, operand=lambda x: x):
    """The steps on one matrix, in 64 bits; `operand` rounds what enters a
    product."""
    a, b, c = coefficients
    X = G.double()
    tall = X.shape[0] > X.shape[1]
    X = X.t() if tall else X
    X = X / (X.square().sum().sqrt() + eps)
    for _ in range(steps):
        x = operand(X)
        S = operand(x @ x.t())
        X = a * X + operand(b * S + c * (S @ S)) @ x
    return X.t() if tall else X


def half(scale):
    def f(x):
        # X and P are stored times 2^8, S times 2^10: only half's subnormals depend on it
        return (x * scale).half().double() / scale
    return f


def check(G, **kw):
    gpu_util.log(f"orthogonalise {tuple(G.shape)} {G.dtype} {kw}")
    X = oz.ozaki25_orthogonalise(G, **kw)
    torch.cuda.synchronize()
    assert X.shape == G.shape and X.dtype == torch.bfloat16
    for x, g in zip(X.reshape(-1, *X.shape[-2:]), G.reshape(-1, *G.shape[-2:])):
        want = exact(g, **kw)
        d = (exact(g, operand=half(256.0), **kw) - want).norm()
        off = (x.double() - want).norm()
        assert off <= 2 * d + (2.0 ** -9 + 1e-5) * want.norm(), (float(off / want.norm()), float(d / want.norm()))
    return X


def gradient(shape, dtype, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    n = lambda *s: torch.randn(s, device="cuda", generator=gen)  # noqa: E731
    low = n(*shape[:-1], 1) * n(*shape[:-2], 1, shape[-1])
    return ((n(*shape) + 0.5 * low) * 1e-3).to(dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("shape", [(4, 128, 128), (2, 64, 200), (2, 200, 64), (3, 129, 257), (3, 257, 129), (1, 7, 5),
                                   (2, 1, 9), (2, 9, 1), (1, 1, 1), (1, 515, 300), (40, 16, 24)])
def test_shapes(shape, dtype):
    check(gradient(shape, dtype))


@pytest.mark.parametrize("shape", [(2, 1024, 512), (1, 512, 1536), (1, 1537, 515), (5, 300, 1000)])
def test_several_tiles(shape):
    check(gradient(shape, torch.float32))


@pytest.mark.parametrize("shape", [(1, 4096, 4096), (3, 2304, 2560)])
def test_large_tiles(shape):
    check(gradient(shape, torch.bfloat16))


def test_one_matrix_and_coefficients():
    G = gradient((96, 160), torch.float32)
    for steps in (1, 2, 9):
        check(G, steps=steps)
    check(G, steps=12, coefficients=(1.5, -0.5, 0.0))
    check(G, steps=8, coefficients=(15 / 8, -10 / 8, 3 / 8), eps=1e-3)


def test_singular_values():
    """Five steps take singular values of 0.01 to 1 of the norm to [0.65, 1.25]
    (the polynomial's own range there, wider by the rounding), and keep the
    singular vectors: X^T G is symmetric to the rounding."""
    gen = torch.Generator(device="cuda").manual_seed(3)
    U = torch.linalg.qr(torch.randn(192, 192, dtype=torch.float64, device="cuda", generator=gen)).Q
    V = torch.linalg.qr(torch.randn(320, 192, dtype=torch.float64, device="cuda", generator=gen)).Q
    s = torch.logspace(-2, 0, 192, dtype=torch.float64, device="cuda")
    s *= 1 / s.norm()
    s = s.clamp(min=0.01)
    G = (U * s @ V.t()).float()
    X = oz.ozaki25_orthogonalise(G, eps=0.0)
    torch.cuda.synchronize()
    got = torch.linalg.svdvals(X.double())
    want = s.clone() / s.norm()
    for _ in range(5):
        want = MUON[0] * want + MUON[1] * want ** 3 + MUON[2] * want ** 5
    assert float(got.min()) > float(want.min()) - 0.02 and float(got.max()) < float(want.max()) + 0.02
    D = U.t() @ X.double() @ V
    off = D - torch.diag(torch.diag(D))
    assert float(off.norm()) < 0.01 * float(D.norm())


@pytest.mark.parametrize("exponent", [-60, -100, 40, 100])
def test_scale_does_not_matter(exponent):
    """Powers of two far outside half's and the squares' float32 range."""
    G = gradient((2, 72, 104), torch.float32)
    want = oz.ozaki25_orthogonalise(G, eps=0.0)
    got = oz.ozaki25_orthogonalise(G * 2.0 ** exponent, eps=0.0)
    torch.cuda.synchronize()
    assert torch.equal(want, got)


def test_zeros_and_nonfinite():
    G = gradient((4, 80, 56), torch.float32)
    G[1] = 0
    G[2, 3, 4] = float("nan")
    G[3, 79, 55] = float("inf")
    X = oz.ozaki25_orthogonalise(G)
    torch.cuda.synchronize()
    assert torch.isfinite(X[0]).all() and not X[1].any() and torch.isnan(X[2]).all() and torch.isnan(X[3]).all()


@pytest.mark.parametrize("pad", [1, 8])
def test_pitches_and_views(pad):
    wide = gradient((3, 70, 90 + pad), torch.bfloat16)
    out = torch.full((3, 71, 90 + pad), 7.0, dtype=torch.bfloat16, device="cuda")
    G = wide[:, :, :90]
    X = oz.ozaki25_orthogonalise(G, X=out[:, :70, :90])
    torch.cuda.synchronize()
    assert torch.equal(X, oz.ozaki25_orthogonalise(G.contiguous()))
    assert bool((out[:, 70:] == 7).all()) and bool((out[:, :, 90:] == 7).all())


@pytest.mark.parametrize("shape", [(2, 128, 128), (1, 300, 520)])
def test_workspace_streams_and_repeats(shape):
    G = gradient(shape, torch.float32)
    want = oz.ozaki25_orthogonalise(G)
    need = oz.ozaki25_orthogonalise_workspace_size(*shape)
    room = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
    other = torch.cuda.Stream()
    torch.cuda.synchronize()
    for kw in (dict(workspace=room), dict(stream=other), dict(stream=other.cuda_stream, workspace=room)):
        got = oz.ozaki25_orthogonalise(G, **kw)
        torch.cuda.synchronize()
        assert torch.equal(got, want)
    with pytest.raises(oz.Ozaki25Error):
        oz.ozaki25_orthogonalise(G, workspace=room[:need - 1])


@pytest.mark.parametrize("shape", [(2, 128, 128), (1, 300, 520)])
def test_in_a_graph(shape):
    G = gradient(shape, torch.float32)
    room = torch.empty(oz.ozaki25_orthogonalise_workspace_size(*shape), dtype=torch.uint8, device="cuda")
    oz.ozaki25_orthogonalise(G, workspace=room)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        X = oz.ozaki25_orthogonalise(G, workspace=room)
    for seed in range(4):
        G.copy_(gradient(shape, torch.float32, seed + 7))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(X, oz.ozaki25_orthogonalise(G))


def test_empty():
    for shape in ((0, 4, 4), (2, 0, 4), (2, 4, 0)):
        assert oz.ozaki25_orthogonalise(torch.empty(shape, device="cuda")).shape == shape
