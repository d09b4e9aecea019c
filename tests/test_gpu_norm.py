"""The root-mean-square norm, its 8-bit output and its gradients against the
formulas in 64 bits.

Sums of squares run over at most 32 elements a thread and then a tree of at most
10 + 15 additions, so they are off by at most 57 roundings of FP32 (U = 2^-24,
relative: the terms have one sign), half of that after the root; the root, the
reciprocal, the division, eps and the two products add at most 6.  35 U in all,
beside the one rounding to the output's type."""
import pytest

import gpu_util
import paper_2609_09095_amd as oz

pytestmark = pytest.mark.gpu
EPS = 1e-6


@pytest.fixture(scope="module", autouse=True)
def gpu():
    gpu_util.require_gpu()


WIDTHS = [1, 7, 8, 9, 64, 127, 128, 129, 200, 256, 500, 512, 1000, 1024, 1031, 2048, 2049, 4096, 4100, 8192, 8200, 11687,
          16384, 20001, 32768]


def case(rows, width, dtype, residual, seed, pad=0, weight=True):
    import eight_util as u
    dt = u.TYPES[dtype]
    X = u.normal((rows, width), dt, seed, 2.0, pad)
    R = u.normal((rows, width), dt, seed + 1, 0.5, pad) if residual else None
    w = (1 + 0.3 * u.normal((width,), u.TYPES["f32"], seed + 2)).to(dt) if weight else None
    return X, R, w


def expected(X, R, w):
    H = X if R is None else (X.float() + R.float()).to(X.dtype)
    h = H.double()
    y = h / (h.square().mean(1, keepdim=True) + EPS).sqrt()
    return H, y if w is None else y * w.double()


def close(got, want, dtype, slack):
    import eight_util as u
    tiny = 2.0 ** -25 if dtype == u.TYPES["f16"] else 0.0  # half a step of the subnormal numbers
    off = (got.double() - want).abs() - want.abs() * (u.half_step(dtype) + slack) - tiny
    assert bool((off <= 0).all()), float(off.max())


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("width", WIDTHS)
def test_norm(width, dtype):
    import torch
    import eight_util as u
    rows = 5 if width > 2048 else 67
    for residual in (False, True):
        X, R, w = case(rows, width, dtype, residual, width, pad=3 if residual else 0, weight=width % 2 == 0)
        H, want = expected(X, R, w)
        got = oz.ozaki25_rms_norm(X, w, residual=R, eps=EPS)
        if residual:
            got, kept = got
            assert torch.equal(kept, H)
        assert got.dtype == X.dtype and got.shape == X.shape
        close(got, want, X.dtype, 35 * u.U)
        out = oz.ozaki25_rms_norm(X, w, residual=R, eps=EPS, quantised=True)
        Q, s = out[:2]
        assert Q.dtype == u.E4M3 and Q.shape == X.shape and s.shape == (-(-width // 128), rows)
        if residual:
            assert torch.equal(out[2], H)
        true = u.spread(u.block_scales(want.float()), rows, width)
        s = u.spread(s, rows, width)
        assert float(((s - true).abs() / true).max()) <= 38 * u.U
        u.assert_e4m3(Q, want / s.double(), 38 * u.U)


@pytest.mark.parametrize("rows", [1, 2, 16, 17, 255, 4097, 70001])
def test_rows(rows):
    """Row counts below and above what the card holds at a time, a norm per head."""
    import eight_util as u
    for width in (64, 100, 512) if rows < 70001 else (64,):
        X, R, w = case(rows, width, "bf16", True, rows)
        H, want = expected(X, R, w)
        Y, _ = oz.ozaki25_rms_norm(X, w, residual=R, eps=EPS)
        close(Y, want, X.dtype, 35 * u.U)


def test_sum_in_place_and_slices():
    """H over X, H over the residual, outputs that are slices: their other columns
    keep their values."""
    import torch
    import eight_util as u
    X, R, w = case(33, 1000, "bf16", True, 5, pad=5)
    H, want = expected(X, R, w)
    for over in ("x", "r"):
        x, r = u.padded(X.clone(), 5, 7.0), u.padded(R.clone(), 5, 7.0)
        h = x if over == "x" else r
        wide = torch.full((33, 1010), 9.0, dtype=torch.bfloat16, device="cuda")
        Y, kept = oz.ozaki25_rms_norm(x, w, residual=r, eps=EPS, Y=wide[:, 4:1004], H=h)
        assert kept is h and torch.equal(h, H)
        close(Y, want, X.dtype, 35 * u.U)
        assert bool((wide[:, :4] == 9).all()) and bool((wide[:, 1004:] == 9).all())
        assert bool((h.as_strided((33, 5), h.stride(), 1000) == 7).all())
        assert torch.equal(r if over == "x" else x, R if over == "x" else X)


def test_values_at_the_ends():
    """Rows of zeros, a NaN, an infinity, the smallest numbers; each stays in its row
    and an 8-bit block that it does not touch keeps its numbers where the row's sum
    is finite."""
    import torch
    import eight_util as u
    X = torch.ones((6, 300), dtype=torch.float32, device="cuda")
    X[0] = 0
    X[1, 5] = float("nan")
    X[2, 200] = float("inf")
    X[3] = 1e-42
    X[4] = 3e4
    w = torch.full((300,), 1.0, device="cuda")
    Y = oz.ozaki25_rms_norm(X, w, eps=EPS)
    want = expected(X, None, w)[1]
    assert bool((Y[0] == 0).all()) and bool(torch.isnan(Y[1]).all())
    assert bool(torch.isnan(Y[2, 200])) and bool((Y[2, :200] == 0).all())
    close(Y[3:], want[3:], torch.float32, 35 * u.U)
    Q, s = oz.ozaki25_rms_norm(X, w, eps=EPS, quantised=True)
    q = Q.float()
    assert bool((q[0] == 0).all()) and bool((s[:, 0] == u.LEAST).all())
    assert bool(torch.isnan(q[1]).all()) and bool(torch.isnan(s[:, 1]).all())
    assert bool(torch.isnan(q[2, 128:256]).all()) and bool((q[2, :128] == 0).all()) and bool(torch.isnan(s[1, 2]))
    assert bool((q[4] == 448).all()) and bool((q[5] == 448).all())
    # a sum of two numbers beyond half's range is an infinity, as half's own addition gives
    h = torch.full((1, 64), 6e4, dtype=torch.float16, device="cuda")
    _, H = oz.ozaki25_rms_norm(h, None, residual=h)
    assert bool(torch.isinf(H).all())


def gradients(dY, H, w, dH):
    h, g = H.double(), dY.double() * (1.0 if w is None else w.double())
    rho = 1 / (h.square().mean(1, keepdim=True) + EPS).sqrt()
    dX = rho * (g - h * rho ** 2 * (g * h).mean(1, keepdim=True))
    return dX if dH is None else dX + dH.double(), (dY.double() * h * rho).sum(0), g, rho


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("width", WIDTHS)
def test_gradients(width, dtype):
    """dX's two terms cancel, so its tolerance goes by their size: the second one's
    mean is off by 57 roundings of the mean of |g h|.  dw by the size of its terms:
    `rows` additions, each term off by 35 U + 2 U."""
    import torch
    import eight_util as u
    rows = 7 if width > 2048 else 131
    for dh in (False, True):
        H, D, w = case(rows, width, dtype, dh, width + 9, pad=1 if dh else 0, weight=width % 3 != 0)
        dY = u.normal((rows, width), H.dtype, width + 5, pad=1 if dh else 0)
        want, dw, g, rho = gradients(dY, H, w, D)
        dX, got = oz.ozaki25_rms_norm_backward(dY, H, w, dH=D, eps=EPS)
        h = H.double().abs()
        size = rho * (g.abs() + h * rho ** 2 * (g * H.double()).abs().mean(1, keepdim=True))
        size = size if D is None else size + D.double().abs()
        tiny = 2.0 ** -25 if H.dtype == torch.float16 else 0.0
        off = (dX.double() - want).abs() - want.abs() * u.half_step(H.dtype) - size * (3 * 35 + 64) * u.U - tiny
        assert bool((off <= 0).all()), float(off.max())
        terms = (dY.double() * H.double() * rho).abs().sum(0)
        assert got.dtype == torch.float32 and bool(((got.double() - dw).abs() <= terms * (rows + 37 + 32) * u.U).all())


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("width", [2100, 8192, 8200, 12288, 12296, 16384, 16400])
def test_gradients_of_wide_rows(width, dtype):
    """More rows than the card holds blocks, so that each goes through several: the sums
    that stay from row to row, the loads ahead, dX in dH's place.  Tolerances as above."""
    import torch
    import eight_util as u
    rows = 700
    H, D, w = case(rows, width, dtype, True, width + 1)
    dY = u.normal((rows, width), H.dtype, width + 2)
    want, dw, g, rho = gradients(dY, H, w, D)
    kept = D.clone()
    dX, got = oz.ozaki25_rms_norm_backward(dY, H, w, dH=kept, dX=kept, eps=EPS)
    assert dX is kept
    size = rho * (g.abs() + H.double().abs() * rho ** 2 * (g * H.double()).abs().mean(1, keepdim=True)) + D.double().abs()
    tiny = 2.0 ** -25 if H.dtype == torch.float16 else 0.0
    off = (dX.double() - want).abs() - want.abs() * u.half_step(H.dtype) - size * (3 * 35 + 64) * u.U - tiny
    assert bool((off <= 0).all()), float(off.max())
    terms = (dY.double() * H.double() * rho).abs().sum(0)
    assert bool(((got.double() - dw).abs() <= terms * (rows + 37 + 32) * u.U).all())
    assert torch.equal(oz.ozaki25_rms_norm_backward(dY, H, w, eps=EPS)[1], got)


@pytest.mark.parametrize("rows", [0, 1, 300, 20000])
def test_gradient_rows(rows):
    """None, one, more than a block and more than the card holds; the same bits twice."""
    import torch
    import eight_util as u
    H, D, w = case(rows, 136, "f32", True, rows)
    dY = u.normal((rows, 136), H.dtype, rows + 5)
    want, dw, g, rho = gradients(dY, H, w, D)
    room = torch.empty((oz.ozaki25_rms_norm_backward_workspace_size(rows, 136),), dtype=torch.uint8, device="cuda")
    dX, got = oz.ozaki25_rms_norm_backward(dY, H, w, dH=D, eps=EPS, workspace=room if rows else None)
    terms = (dY.double() * H.double() * rho).abs().sum(0)
    assert bool(((got.double() - dw).abs() <= terms * (min(rows, 400) + 128) * u.U).all())
    # a block's rows one after the other (at most 400 here), then the blocks'
    again = oz.ozaki25_rms_norm_backward(dY, H, w, dH=D, eps=EPS)
    assert torch.equal(dX, again[0]) and torch.equal(got, again[1])


def test_gradients_in_place():
    import torch
    import eight_util as u
    H, D, w = case(50, 777, "bf16", True, 3)
    dY = u.normal((50, 777), H.dtype, 4)
    dX, dw = oz.ozaki25_rms_norm_backward(dY, H, w, dH=D)
    for over in ("dY", "dH"):
        t = {"dY": dY.clone(), "dH": D.clone()}
        a, b = oz.ozaki25_rms_norm_backward(t["dY"], H, w, dH=t["dH"], dX=t[over])
        assert a is t[over] and torch.equal(a, dX) and torch.equal(b, dw)


def test_gradients_against_differences():
    """Central differences of sum(Y dY) in FP64 along random directions against the
    gradients (32-bit inputs): the difference quotient with steps of 1e-5 is off by
    about 1e-9 of its terms."""
    import torch
    import eight_util as u
    H, _, w = case(9, 70, "f32", False, 8)
    dY = u.normal((9, 70), H.dtype, 9)
    dX, dw = oz.ozaki25_rms_norm_backward(dY, H, w, eps=EPS)

    def f(h, v):
        return float((h / (h.square().mean(1, keepdim=True) + EPS).sqrt() * v * dY.double()).sum())

    for seed in range(4):
        a, b = u.normal((9, 70), torch.float32, 20 + seed).double(), u.normal((70,), torch.float32, 30 + seed).double()
        h, v, t = H.double(), w.double(), 1e-5
        num = (f(h + t * a, v) - f(h - t * a, v)) / (2 * t)
        assert abs(num - float((dX.double() * a).sum())) < 1e-6 * float((dX.double() * a).abs().sum())
        num = (f(h, v + t * b) - f(h, v - t * b)) / (2 * t)
        assert abs(num - float((dw.double() * b).sum())) < 1e-6 * float((dw.double() * b).abs().sum())
