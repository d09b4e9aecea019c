"""The product of e4m3 matrices with scales of blocks of 128, in every form, against
the same sum in 64 bits.

The products of two e4m3 numbers are exact in FP32 (U = 2^-24).  For a 16-bit output
the matrix cores add eight products of neighbouring depths as whole multiples of
2^-13 of the largest: each is off by one such multiple at most, so a block is off by
at most 8 2^-13 times the largest product of each eight, and no more than that times
the sum of magnitudes: 2^-10.  (Sums stray from that by far less; a wrong number, scale
or place is off by more.)  For an FP32 output the 128 products of a block are added
with at most 128 roundings relative to the sum of the magnitudes.  In both the two
scales' product rounds once, and each block's share is added with one rounding:
(1 + blocks) U, up to eleven more for joins of parts of the depth, beside the
output's own rounding."""
import pytest

import gpu_util
import paper_2609_09095_amd as oz

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def gpu():
    gpu_util.require_gpu()


def operands(rows, n, k, squares, seed, layout="padded", spread=2.0):
    """e4m3 operands with scales that differ, and what they stand for in 64 bits.
    layout: rows on 16 bytes with NaN behind their ends, `tight`, or at an odd
    address and pitch."""
    import torch
    import eight_util as u

    def one(v, seed, sq):
        X = u.normal((v, k), torch.float32, seed) * torch.exp(spread * u.normal((v, 1), torch.float32, seed + 1) / 2)
        Q, s = u.quantised(X, sq)
        V = Q.double() * u.spread(s, v, k, sq).double()
        if layout == "padded":
            Q = u.e4m3_rows(Q, -k % 16)
        elif layout == "odd":
            Q = u.e4m3_rows(Q, 5)
            flat = torch.full((Q.stride(0) * v + 3,), 0x7f, dtype=torch.uint8, device="cuda")
            at = flat[3:].as_strided((v, k), (Q.stride(0), 1))
            at.copy_(Q.view(torch.uint8))
            Q = at.view(u.E4M3)
        return Q, s, V

    return one(rows, seed, False), one(n, seed + 7, squares)


def check(rows, n, k, squares, dtype, seed=0, layout="padded", **kw):
    import torch
    import eight_util as u
    (A, a, VA), (B, b, VB) = operands(rows, n, k, squares, seed, layout)
    Y = oz.ozaki25_scaled_matmul(A, a, B, b, squares=squares, out_dtype=u.TYPES[dtype], **kw)
    want, size = VA @ VB.t(), VA.abs() @ VB.t().abs()
    tiny = 2.0 ** -25 if dtype == "f16" else 0.0
    allowed = size * ((128 + 12 + -(-k // 128)) * u.U if dtype == "f32" else 2.0 ** -10)
    off = (Y.double() - want).abs() - want.abs() * u.half_step(Y.dtype) - allowed - tiny
    if dtype == "f16":
        # half rounds from 65520 on (65504 and half a step, 16) to an infinity of the sign:
        # it has to where all of the sum's range lies beyond, and may where some does
        most = 65520.0
        beyond = torch.isinf(Y) & (torch.sign(Y.double()) == torch.sign(want)) & (want.abs() + allowed >= most)
        assert bool(beyond[want.abs() - allowed >= most].all())
        off = torch.where(beyond, 0.0, off)
    assert Y.shape == (rows, n) and bool((off <= 0).all()), (float(off.max()), int((off > 0).sum()))
    return Y


FEW = [(1, 1, 1), (1, 16, 128), (1, 17, 129), (2, 1000, 1111), (16, 48, 4096), (17, 40, 300), (32, 130, 256), (33, 100, 77),
       (48, 256, 1500), (41, 1000, 1111), (49, 130, 300), (64, 256, 1500), (1, 4096, 4096)]
TILES = [(65, 64, 128), (65, 1, 1), (100, 70, 15), (128, 128, 129), (200, 129, 1000), (333, 1000, 1111), (500, 300, 2048),
         (256, 256, 16), (97, 333, 640)]
MANY = [(2000, 2048, 300), (2049, 2050, 257), (4096, 4096, 128), (4100, 4000, 1000), (3300, 2050, 1300)]


@pytest.mark.parametrize("squares", [True, False])
@pytest.mark.parametrize("layout", ["padded", "tight", "odd"])
@pytest.mark.parametrize("rows,n,k", FEW + TILES)
def test_products(rows, n, k, layout, squares):
    for i, dtype in enumerate(("bf16", "f16", "f32")):
        check(rows, n, k, squares, dtype, rows + n + k + i, layout)


@pytest.mark.parametrize("squares", [True, False])
@pytest.mark.parametrize("rows,n,k", MANY)
def test_many_tiles(rows, n, k, squares):
    for dtype in ("bf16", "f32"):
        check(rows, n, k, squares, dtype, 3, "padded")
    check(rows, n, k, squares, "f16", 4, "odd")


@pytest.mark.parametrize("squares", [True, False])
@pytest.mark.parametrize("rows,n,k", [(100, 70, 3075), (65, 130, 3200), (285, 128, 7355), (1100, 1030, 8200), (40, 33, 6145)])
def test_depths_in_parts(rows, n, k, squares):
    """Few tiles of a long depth: its parts' sums, in a workspace given or not."""
    import torch
    room = oz.ozaki25_scaled_matmul_workspace_size(rows, n, k)
    assert room > 0
    for dtype, layout in (("bf16", "padded"), ("f32", "tight"), ("f16", "odd")):
        Y = check(rows, n, k, squares, dtype, k, layout)
        again = check(rows, n, k, squares, dtype, k, layout, workspace=torch.full((room,), 0xff, dtype=torch.uint8, device="cuda"))
        assert torch.equal(Y, again)


def test_large_tiles_of_every_depth():
    """Whole and cut last stages behind one, two, three and more whole ones."""
    for k in (1, 127, 128, 130, 255, 256, 258, 384, 400, 513):
        check(4096, 3600, k, True, "bf16", k)


@pytest.mark.parametrize("rows", [3, 70, 3000])
def test_no_depth(rows):
    import torch
    import eight_util as u
    A, B = torch.empty((rows, 0), dtype=u.E4M3, device="cuda"), torch.empty((90, 0), dtype=u.E4M3, device="cuda")
    for squares in (True, False):
        Y = torch.full((rows, 90), 5.0, device="cuda")
        oz.ozaki25_scaled_matmul(A, torch.empty((0, rows), device="cuda"), B, torch.empty((1, 0) if squares else (0, 90), device="cuda"),
                                 squares=squares, Y=Y)
        assert bool((Y == 0).all())


def test_empty():
    import torch
    import eight_util as u
    A, B = torch.empty((0, 300), dtype=u.E4M3, device="cuda"), torch.zeros((90, 300), device="cuda").to(u.E4M3)
    assert oz.ozaki25_scaled_matmul(A, torch.empty((3, 0), device="cuda"), B, torch.ones((1, 3), device="cuda")).shape == (0, 90)


@pytest.mark.parametrize("rows", [5, 60, 200, 2500])
def test_outputs_and_scales_in_slices(rows):
    """Pitches of scales and outputs; what lies beside the output stays."""
    import torch
    import eight_util as u
    (A, a, VA), (B, b, VB) = operands(rows, 300, 500, False, rows)
    a = u.padded(a, 3, float("nan"))
    b = u.padded(b, 5, float("nan"))
    for dtype in (torch.bfloat16, torch.float32):
        wide = torch.full((rows, 311), 3.0, dtype=dtype, device="cuda")
        Y = oz.ozaki25_scaled_matmul(A, a, B, b, squares=False, Y=wide[:, 5:305])
        want = VA @ VB.t()
        assert float((Y.double() - want).norm() / want.norm()) < u.half_step(dtype) + 1e-6
        assert bool((wide[:, :5] == 3).all()) and bool((wide[:, 305:] == 3).all())


@pytest.mark.parametrize("rows", [4, 40, 150, 2300])
def test_not_a_number_stays_in_its_row(rows):
    """A NaN scale or number of one row (column) reaches that row (column) alone."""
    import torch
    import eight_util as u
    for squares in (True, False):
        (A, a, VA), (B, b, VB) = operands(rows, 270, 400, squares, rows)
        a[2, rows - 1] = float("nan")
        A.view(torch.uint8)[1, 399] = 0x7f
        Y = oz.ozaki25_scaled_matmul(A, a, B, b, squares=squares)
        bad = torch.isnan(Y).all(1)
        assert bool(bad[rows - 1]) and bool(bad[1]) and int(torch.isnan(Y).any(1).sum()) == 2
        a[2, rows - 1], A.view(torch.uint8)[1, 399] = 1.0, 0
        b[(1, 0) if squares else (0, 135)] = float("inf")
        Y = oz.ozaki25_scaled_matmul(A, a, B, b, squares=squares)
        fine = torch.isfinite(Y).all(0)
        cols = torch.arange(270, device="cuda")
        assert torch.equal(fine, ~((cols >= 128) & (cols < 256)) if squares else cols != 135)


def test_same_bits_twice_and_rows_alone():
    import torch
    (A, a, _), (B, b, _) = operands(700, 500, 3000, True, 1)
    Y = oz.ozaki25_scaled_matmul(A, a, B, b)
    assert torch.equal(Y, oz.ozaki25_scaled_matmul(A, a, B, b))


def test_a_projection_and_its_gradients():
    """Forward, input's and weights' gradient of Y = X W^T from one quantisation each,
    against the products of the numbers that the operands stand for."""
    import torch
    import eight_util as u
    rows, n, k = 300, 200, 410
    X, W = u.normal((rows, k), torch.bfloat16, 1), u.normal((n, k), torch.float32, 2, k ** -0.5)
    dY = u.normal((rows, n), torch.bfloat16, 3)
    w, ws, wt, wts = oz.ozaki25_quantise(W, squares=True, layout="both")
    x, xs, xt, xts = oz.ozaki25_quantise(X, layout="both")
    y, ys, yt, yts = oz.ozaki25_quantise(dY, layout="both")
    Wv = w.double() * u.spread(ws, n, k, True).double()
    Xv, Xt = x.double() * u.spread(xs, rows, k).double(), xt.double() * u.spread(xts, k, rows).double()
    Yv, Yt = y.double() * u.spread(ys, rows, n).double(), yt.double() * u.spread(yts, n, rows).double()
    assert torch.equal(wt.t().float(), w.float()) and torch.equal(wts.t(), ws)
    for got, want in ((oz.ozaki25_scaled_matmul(x, xs, w, ws), Xv @ Wv.t()),
                      (oz.ozaki25_scaled_matmul(y, ys, wt, wts), Yv @ Wv),
                      (oz.ozaki25_scaled_matmul(yt, yts, xt, xts, squares=False, out_dtype=torch.float32), Yt @ Xt.t())):
        assert float((got.double() - want).norm() / want.norm()) < u.half_step(got.dtype) + 1e-6
    # and near those of the unrounded operands: both roundings of e4m3 at most 2^-4 each
    for got, want in ((oz.ozaki25_scaled_matmul(x, xs, w, ws), X.double() @ W.double().t()),
                      (oz.ozaki25_scaled_matmul(y, ys, wt, wts), dY.double() @ W.double()),
                      (oz.ozaki25_scaled_matmul(yt, yts, xt, xts, squares=False), dY.double().t() @ X.double())):
        assert float((got.double() - want).norm() / want.norm()) < 2 * 2.0 ** -4


@pytest.mark.parametrize("rows", [3, 20, 80])
def test_pitches_beyond_the_tiles_offsets(rows):
    """Rows 2^22 bytes and more apart."""
    import torch
    import eight_util as u
    (A, a, VA), (B, b, VB) = operands(rows, 90, 300, True, rows)
    for pitch in (1 << 22, (1 << 22) + 3):
        wide = torch.empty(((rows - 1) * pitch + 300,), dtype=torch.uint8, device="cuda")
        far = wide.as_strided((rows, 300), (pitch, 1))
        far.copy_(A.view(torch.uint8))
        Y = oz.ozaki25_scaled_matmul(far.view(u.E4M3), a, B, b)
        want, size = VA @ VB.t(), VA.abs() @ VB.t().abs()
        assert bool(((Y.double() - want).abs() <= want.abs() * 2.0 ** -8 + size * 2.0 ** -10).all())


def test_large_offsets():
    """Rows of A and Y beyond 2^32 bytes."""
    import torch
    import eight_util as u
    rows, n, k = (1 << 21) + 70, 1100, 2064
    A = torch.zeros((rows, k), dtype=torch.uint8, device="cuda").view(u.E4M3)
    (T, a, V), (B, b, VB) = operands(200, n, k, True, 5)
    A.view(torch.uint8)[-200:] = T.view(torch.uint8)
    s = torch.ones((a.shape[0], rows), device="cuda")
    s[:, -200:] = a
    Y = oz.ozaki25_scaled_matmul(A, s, B, b)
    want = V @ VB.t()
    assert float((Y[-200:].double() - want).norm() / want.norm()) < 2.0 ** -8 and bool((Y[:5000] == 0).all())
