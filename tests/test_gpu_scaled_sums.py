"""What the 8-bit products keep of their sums, in every form.

Small whole numbers (products up to 9) with scales that are powers of two: every partial
sum is a multiple of 1/2 below 2^23, and an eight's products lie within 13 bits of each
other, so all sums are exact however they are grouped, and a result is the exact sum
rounded once.  One product lost, doubled or out of place shows.

Large products that cancel: an FP32 output's sums are exact as long as they are whole
numbers below 2^24.  For a 16-bit output each eight neighbouring depths (8 i .. 8 i + 7)
may be off by 8 2^-13 of its largest product; beside that at most one FP32 rounding for
each eight and each block, relative to the sum of magnitudes, and the output's own."""
import pytest

import eight_routes
import gpu_util
import paper_2609_09095_amd as oz

pytestmark = pytest.mark.gpu
E = 2.0 ** -24


@pytest.fixture(scope="module", autouse=True)
def gpu():
    gpu_util.require_gpu()


def laid(Q, layout):
    """Rows on 16 bytes ("padded"), on 4 but not on 16 ("words"), or at odd places."""
    import torch
    import eight_util as u
    v, k = Q.shape
    if layout == "padded":
        return u.e4m3_rows(Q, -k % 16)
    first, pitch = (4, -(-k // 16) * 16 + 4) if layout == "words" else (3, (k + 4) // 2 * 2 + 1)
    flat = torch.full((pitch * v + first,), 0x7f, dtype=torch.uint8, device="cuda")
    at = flat[first:].as_strided((v, k), (pitch, 1))
    at.copy_(Q.view(torch.uint8))
    return at.view(u.E4M3)


def powers(shape, lo, hi, seed):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return 2.0 ** torch.randint(lo, hi + 1, shape, device="cuda", generator=gen).float()


def wholes(shape, most, seed):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(-most, most + 1, shape, device="cuda", generator=gen).float()


def scales(rows, n, k, squares, seed):
    blocks = lambda x: -(-x // 128)  # noqa: E731
    return powers((blocks(k), rows), 0, 2, seed), powers((blocks(n), blocks(k)) if squares else (blocks(k), n), -1, 1, seed + 1)


def values(Q, s, squares):
    import eight_util as u
    return Q.double() * u.spread(s, *Q.shape, squares).double()


EXACT = [
    # rows, n, k, layout, the form of a 16-bit output with squares, of another
    (3, 500, 5000, "padded", ("few16", "", 1), ("few16", "", 1)), (3, 500, 3000, "odd", ("few16", "", 1), ("few16", "", 1)),
    (3, 500, 5000, "words", ("few16", "", 1), ("few16", "", 1)), (3, 500, 5300, "odd", ("small", "masked", 5), ("small", "masked", 5)),
    (8, 500, 4097, "odd", ("small", "masked", 4), ("small", "masked", 4)), (8, 70, 4095, "odd", ("few16", "", 1), ("few16", "", 1)),
    (16, 70, 3201, "odd", ("small", "masked", 3), ("small", "masked", 3)), (30, 300, 4000, "odd", ("small", "masked", 4), ("small", "masked", 4)),
    (48, 130, 4095, "odd", ("small", "masked", 4), ("small", "masked", 4)), (33, 200, 2000, "odd", ("small", "masked", 1), ("small", "masked", 1)),
    (30, 300, 4000, "words", ("few32", "", 1), ("few32", "", 1)), (48, 130, 4095, "words", ("few48", "", 1), ("few48", "", 1)),
    (49, 130, 4095, "words", ("small", "masked", 4), ("small", "masked", 4)),
    (30, 300, 4000, "padded", ("few32", "", 1), ("few32", "", 1)), (45, 300, 4000, "padded", ("few48", "", 1), ("few48", "", 1)),
    (45, 70, 5000, "padded", ("small", "dma", 5), ("small", "dma", 5)), (45, 70, 5000, "odd", ("small", "masked", 5), ("small", "masked", 5)),
    (300, 200, 2000, "padded", ("small", "dma", 1), ("small", "dma", 1)),
    (300, 200, 2000, "odd", ("small", "masked", 1), ("small", "masked", 1)),
    (1100, 1030, 8200, "padded", ("middle", "dma", 8), ("middle", "dma", 8)),
    (1100, 1030, 8200, "odd", ("middle", "masked", 8), ("middle", "masked", 8)),
    (2000, 1800, 1500, "padded", ("middle", "dma", 1), ("middle", "dma", 1)),
    (4096, 3600, 4100, "odd", ("middle", "masked", 1), ("middle", "masked", 1)),
    (4096, 3600, 4100, "padded", ("large", "dma", 1), ("tall", "dma", 1)),
]


@pytest.mark.parametrize("squares", [True, False])
@pytest.mark.parametrize("rows,n,k,layout,form,other", EXACT)
def test_whole_numbers_are_exact(rows, n, k, layout, form, other, squares):
    import torch
    import eight_util as u
    A, B = wholes((rows, k), 3, rows).to(u.E4M3), wholes((n, k), 3, n + 1).to(u.E4M3)
    a, b = scales(rows, n, k, squares, k)
    want = values(A, a, False) @ values(B, b, squares).t()
    assert float(want.abs().max()) < 32768.0  # in half's range
    A, B = laid(A, layout), laid(B, layout)
    for dtype in ("bf16", "f16", "f32"):
        assert eight_routes.scaled_route(rows, n, k, squares, dtype, A, B) == (form if squares and dtype != "f32" else other)
        Y = oz.ozaki25_scaled_matmul(A, a, B, b, squares=squares, out_dtype=u.TYPES[dtype])
        assert torch.equal(Y, want.to(u.TYPES[dtype])), (dtype, int((Y != want.to(u.TYPES[dtype])).sum()))
        # in a workspace of the stated size, which holds anything
        room = torch.full((oz.ozaki25_scaled_matmul_workspace_size(rows, n, k),), 0xff, dtype=torch.uint8, device="cuda")
        assert torch.equal(oz.ozaki25_scaled_matmul(A, a, B, b, squares=squares, out_dtype=u.TYPES[dtype], workspace=room), Y)


def cancelling(rows, n, k, seed):
    """Whole numbers up to 1, and in every second eight a pair 448 448 and -448 448."""
    import torch
    A, B = wholes((rows, k), 1, seed), wholes((n, k), 1, seed + 1)
    for g in range(0, k - 7, 16):
        i, j = g + g // 16 % 7, g + g // 16 % 7 + 1
        A[:, i] = A[:, j] = B[:, i] = 448.0
        B[:, j] = -448.0
    return A, B, torch.ones(-(-k // 128), rows, device="cuda"), torch.ones(-(-k // 128), n, device="cuda")


def largest_of_eights(A, B):
    """The sum over the eights of depths of their largest product."""
    import torch
    P = torch.zeros((A.shape[0], B.shape[0]), dtype=torch.float64, device="cuda")
    for g in range(0, A.shape[1], 8):
        P += (A[:, None, g:g + 8] * B[None, :, g:g + 8]).abs().amax(2)
    return P


SUMS = [(1, 33, 700, "padded"), (16, 40, 1000, "odd"), (25, 100, 1000, "padded"), (48, 64, 400, "padded"), (48, 64, 400, "odd"),
        (70, 70, 3500, "padded"), (200, 130, 640, "odd"), (4000, 3500, 400, "padded"), (4000, 3500, 400, "odd")]


@pytest.mark.parametrize("rows,n,k,layout", SUMS)
def test_fp32_outputs_keep_what_cancelling_products_leave(rows, n, k, layout):
    import torch
    import eight_util as u
    A, B, a, b = cancelling(rows, n, k, rows)
    Y = oz.ozaki25_scaled_matmul(laid(A.to(u.E4M3), layout), a, laid(B.to(u.E4M3), layout), b, squares=False, out_dtype=torch.float32)
    want = A.double() @ B.double().t()
    assert float(want.abs().max()) > 0 and torch.equal(Y.double(), want)


@pytest.mark.parametrize("kind", ["cancelling", "bytes"])
@pytest.mark.parametrize("rows,n,k,layout", SUMS)
def test_eights_of_16_bit_outputs(rows, n, k, layout, kind):
    """Within the stated bound, for products that cancel and for every finite byte."""
    import torch
    import eight_util as u
    if kind == "cancelling":
        A, B, a, b = cancelling(rows, n, k, rows + 1)
        A, B = A.to(u.E4M3), B.to(u.E4M3)
    else:
        gen = torch.Generator(device="cuda").manual_seed(rows)
        A, B = (torch.randint(0, 256, (v, k), device="cuda", generator=gen).to(torch.uint8) for v in (rows, n))
        A, B = (torch.where((v & 0x7f) == 0x7f, 0x80, v).view(u.E4M3) for v in (A, B))
        a, b = torch.full((-(-k // 128), rows), 2.0 ** -9, device="cuda"), torch.ones(-(-k // 128), n, device="cuda")
    some = torch.randperm(rows, generator=torch.Generator().manual_seed(1))[:60].cuda()
    cols = torch.randperm(n, generator=torch.Generator().manual_seed(2))[:60].cuda()
    V, W = values(A, a, False)[some], values(B, b, False)[cols]
    want, size = V @ W.t(), V.abs() @ W.abs().t()
    allowed = largest_of_eights(V, W) * (8 * 2.0 ** -13) + size * ((k // 8 + 1 + 2 * (-(-k // 128)) + 8) * E)
    for dtype in (torch.bfloat16, torch.float16):
        Y = oz.ozaki25_scaled_matmul(laid(A, layout), a, laid(B, layout), b, squares=False, out_dtype=dtype)
        Y = Y[some][:, cols].double()
        assert float((want.abs() + allowed).max()) < 65504
        tiny = 2.0 ** -25 if dtype == torch.float16 else 0.0
        off = (Y - want).abs() - allowed - (want.abs() + allowed) * u.half_step(dtype) - tiny
        assert bool((off <= 0).all()), float(off.max())


@pytest.mark.parametrize("first", [0, 40, 120, 200])
@pytest.mark.parametrize("rows", [16, 40, 256, 4096])
def test_only_its_own_eight_loses_to_a_large_product(rows, first):
    """1 at one depth beside a pair that cancels at depths `first` and `first` + 1: exact
    at every depth of another eight, in an FP32 output at all."""
    import torch
    import eight_util as u
    k, n = 256, 3600 if rows == 4096 else 50
    at = torch.arange(rows, device="cuda") % k if rows >= k else (torch.arange(rows, device="cuda") + first) % k
    A, B = torch.zeros((rows, k), device="cuda"), torch.ones((n, k), device="cuda")
    A[torch.arange(rows, device="cuda"), at] = 1.0
    A[:, first] = A[:, first + 1] = B[:, first] = 448.0
    B[:, first + 1] = -448.0
    want = (~((at == first) | (at == first + 1))).double()[:, None].expand(rows, n)
    ones = torch.ones(2, rows, device="cuda"), torch.ones(-(-n // 128), 2, device="cuda")
    beside = (at // 8 == first // 8)[:, None].expand(rows, n)
    for dtype in u.TYPES.values():
        Y = oz.ozaki25_scaled_matmul(A.to(u.E4M3), ones[0], B.to(u.E4M3), ones[1], out_dtype=dtype).double()
        if dtype == torch.float32:
            assert torch.equal(Y, want)
        else:
            assert torch.equal(Y[~beside], want[~beside])
            assert bool(((Y - want).abs()[beside] <= 448.0 * 448 * 8 * 2.0 ** -13).all())


@pytest.mark.parametrize("squares", [True, False])
@pytest.mark.parametrize("rows,n,k", [(4096, 3600, 4096), (2048, 2048, 4096), (300, 300, 8192), (16, 1000, 8192)])
def test_long_sums_of_normal_numbers(rows, n, k, squares):
    """Normwise.  An eight drops seven rests below 2^-13 of its largest product, which is
    about 2.5 times a product's size: of k / 8 eights, independent in sign, at most
    sqrt(7 / 8) 2.5 2^-13 < 2^-11.7 of the result's norm, less than half's own rounding
    (2^-11) to which it adds; one product lost in each sum of 8192 would be 2^-6.5."""
    import torch
    import eight_util as u
    (A, a), (B, b) = u.quantised(u.normal((rows, k), torch.float32, 1)), u.quantised(u.normal((n, k), torch.float32, 2), squares)
    want = values(A, a, False) @ values(B, b, squares).t()
    for dtype in (torch.bfloat16, torch.float16):
        Y = oz.ozaki25_scaled_matmul(A, a, B, b, squares=squares, out_dtype=dtype).double()
        assert float((Y - want).norm() / want.norm()) < u.half_step(dtype) + 2.0 ** -11.7
