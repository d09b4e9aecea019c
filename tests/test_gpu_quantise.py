"""Matrices in 8 bits: scales and numbers against the stated rule, in every
layout, over odd sizes, pitches and the ends of the range."""
import pytest

import gpu_util
import paper_2609_09095_amd as oz

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def gpu():
    gpu_util.require_gpu()


def check(X, Q, s, squares):
    """Scales are the FP32 quotients themselves (one correctly rounded division; a
    step, 2^-23, is allowed); numbers are within half a step of x / s."""
    import torch
    import eight_util as u
    assert Q.dtype == u.E4M3 and Q.shape == X.shape
    true = u.block_scales(X, squares)
    assert s.shape == true.shape and torch.equal(torch.isnan(s), torch.isnan(true))
    assert bool(((s - true).abs() <= true * 2 * u.U).logical_or(torch.isnan(true)).all())
    u.assert_e4m3(Q, X.double() / u.spread(s, *X.shape, squares).double())


SIZES = [(1, 1), (1, 128), (1, 4096), (7, 130), (128, 128), (129, 127), (130, 300), (256, 1000), (777, 1031), (300, 8), (2000, 65)]


@pytest.mark.parametrize("squares", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("rows,cols", SIZES)
def test_layouts(rows, cols, dtype, squares):
    import torch
    import eight_util as u
    X = u.normal((rows, cols), u.TYPES[dtype], rows + cols, 0.7, pad=rows % 3)
    Q, s, QT, sT = oz.ozaki25_quantise(X, squares=squares, layout="both")
    check(X, Q, s, squares)
    check(X.t(), QT, sT, squares)
    for layout, want in (("rows", (Q, s)), ("columns", (QT, sT))):
        got = oz.ozaki25_quantise(X, squares=squares, layout=layout)
        assert len(got) == 2 and all(torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))
                                     for a, b in zip(got, want))


@pytest.mark.parametrize("squares", [False, True])
def test_stacks(squares):
    """Matrices of a stack are apart, also where the stack is a slice."""
    import torch
    import eight_util as u
    full = u.normal((5, 200, 150), torch.float32, 1)
    X = full[1:4, :150, 10:140]
    got = oz.ozaki25_quantise(X, squares=squares, layout="both")
    for i in range(3):
        alone = oz.ozaki25_quantise(X[i], squares=squares, layout="both")
        assert all(torch.equal(a[i].contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))
                   for a, b in zip(got, alone))
        check(X[i], got[0][i], got[1][i], squares)


@pytest.mark.parametrize("squares", [False, True])
def test_ends_of_the_range(squares):
    """Zeros, numbers below the least scale, the largest ones, NaN and infinities:
    a block with one of those is NaN and its neighbours are not."""
    import torch
    X = torch.zeros((300, 400), device="cuda")
    X[:, 128:256] = 3e38
    X[5, 130] = -3.4e38
    X[140:, 256:384] = torch.linspace(1e-44, 1e-38, 128, device="cuda")
    X[2, 390] = float("nan")
    X[280, 140] = float("inf")
    Q, s, QT, sT = oz.ozaki25_quantise(X, squares=squares, layout="both")
    check(X, Q, s, squares)
    check(X.t(), QT, sT, squares)
    assert bool((Q[:, :128].float() == 0).all())
    for dtype in (torch.bfloat16, torch.float16):
        Y = torch.zeros((3, 200), dtype=dtype, device="cuda")
        Y[0, 0], Y[1, 199], Y[2] = torch.finfo(dtype).max, torch.finfo(dtype).tiny / 4, float("-inf")
        Q, s = oz.ozaki25_quantise(Y, squares=squares)
        check(Y, Q, s, squares)


def test_every_number():
    """A block that holds every e4m3 number at a power of two gives them back."""
    import torch
    import eight_util as u
    bytes_ = torch.arange(256, dtype=torch.int32, device="cuda").to(torch.uint8)
    want = bytes_.view(u.E4M3)
    finite = ~torch.isnan(want.float())
    want = want[finite]
    for scale in (1.0, 2.0 ** -20, 2.0 ** 30):
        X = torch.full((2, 128), 448.0 * scale, device="cuda")
        X[0, 1:] = want[:127].float() * scale
        X[1, 1:128] = want[127:].float()[:127] * scale
        Q, s = oz.ozaki25_quantise(X)
        assert bool((s == scale).all())
        assert torch.equal(Q[0, 1:].float(), want[:127].float()) and torch.equal(Q[1, 1:].float(), want[127:].float()[:127])


def test_rows_are_laid_out_on_16_bytes():
    import torch
    X = torch.ones((5, 37), device="cuda")
    Q, _, QT, _ = oz.ozaki25_quantise(X, layout="both")
    assert Q.stride() == (48, 1) and QT.stride() == (16, 1) and Q.data_ptr() % 16 == 0


def test_large_offsets():
    """A matrix whose bytes pass 2^32."""
    import torch
    rows, cols = (1 << 20) + 3, 4104
    X = torch.zeros((rows, cols), dtype=torch.bfloat16, device="cuda")
    X[-2] = torch.arange(cols, device="cuda").to(torch.bfloat16)
    Q, s = oz.ozaki25_quantise(X)
    check(X[-130:], Q[-130:], s[:, -130:].contiguous(), False)
    assert bool((Q[:1000].view(torch.uint8) == 0).all())
