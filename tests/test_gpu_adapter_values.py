"""Values at the ends of their types' ranges in the shared projection with
adapters: small and large s X A^T, infinities in scales, activations and the
rows' own adapters, in every form that rows can take.

Tolerance: as in the tests of the operator, but the two 16-bit numbers that
s X A^T becomes in tiles keep 2^-22 of it in half, at a power of two of their
row's own that puts the row's largest at 2^14 or above, where the least
difference of two numbers is 2^-24: 2^-39 of the row's largest.
"""
import pytest
import torch

import gpu_util
import paper_2609_09095_amd as oz
from half_routes import LARGE, SMALL, adapter_of
from test_gpu_adapter import mixed
from test_gpu_grouped import TINY, UNIT, draw

pytestmark = pytest.mark.gpu

BF, HALF = torch.bfloat16, torch.float16
# rows, n, k: the few-row form; tiles behind products X A^T of single rows; the
# same with operands off 16 bytes; tiles behind products X A^T in tiles
FORMS = [(20, 136, 256, None), (700, 520, 256, SMALL), (700, 520, 257, SMALL), (1100, 520, 256, SMALL)]


@pytest.fixture(scope="module", autouse=True)
def gpu():
    gpu_util.require_gpu()


def takes(rows, n, k, adapters, rank, tile):
    assert adapter_of(rows, n, k, adapters, rank) == (tile, rows if tile is None else 0)
    gpu_util.log(f"adapter rows={rows} n={n} k={k} adapters={adapters} rank={rank}")


def call(*a):
    Y = oz.ozaki25_adapter_matmul(*a)
    torch.cuda.synchronize()
    return Y


def ids_of(rows, adapters):
    return torch.as_tensor(mixed(rows, adapters), dtype=torch.int32, device="cuda")


def reference(X, W, ids, A, B, scales):
    """(Y, bound) in 64 bits."""
    Y, size = X.double() @ W.double().t(), X.double().abs() @ W.double().abs().t()
    low, floor = (2.0 ** -16, 0.0) if X.dtype == BF else (2.0 ** -22, 2.0 ** -39)
    err = torch.zeros_like(Y)
    for a in range(A.shape[0]):
        at = torch.nonzero(ids == a).flatten()
        if len(at) == 0:
            continue
        s, b = float(scales[a]), B[a].double()
        h = s * (X[at].double() @ A[a].double().t())
        hs = abs(s) * (X[at].double().abs() @ A[a].double().abs().t())
        Y[at] += h @ b.t()
        size[at] += hs @ b.abs().t()
        err[at] += (low * h.abs() + floor * h.abs().amax(1, keepdim=True)) @ b.abs().t()
    u = UNIT[X.dtype]
    return Y, ((X.shape[1] + 2 * A.shape[1] + 8) * 2.0 ** -23 * size + err) * (1 + u) + u * Y.abs() + TINY[X.dtype]


def close(got, want, bound):
    bad = ~((got.double() - want).abs() <= bound)
    assert not bad.any(), (int(bad.sum()), float(((got.double() - want).abs() / bound).nan_to_num(1e30).max()))


@pytest.mark.parametrize("dtype", [BF, HALF])
@pytest.mark.parametrize("exponent", [-30, -18, -10, 0, 14, 17, 21])
@pytest.mark.parametrize("rows, n, k, tile", FORMS)
def test_range_of_the_inner_product(dtype, exponent, rows, n, k, tile):
    """s X A^T of about 2^exponent beside a B that brings the outputs back: the
    outputs are in range whatever the inner product is."""
    takes(rows, n, k, 3, 24, tile)
    X, W, ids = draw((rows, k), dtype, 1), torch.zeros((n, k), dtype=dtype, device="cuda"), ids_of(rows, 3)
    A, B = draw((3, 24, k), dtype, 2) * k ** -0.5, draw((3, n, 24), dtype, 3) * 2.0 ** min(max(-exponent, -12), 12)
    scales = torch.tensor([0.5, 1.0, -1.5], device="cuda") * 2.0 ** exponent
    close(call(X, W, ids, A, B, scales), *reference(X, W, ids, A, B, scales))


@pytest.mark.parametrize("dtype", [BF, HALF])
def test_rows_of_a_call_in_both_forms(dtype):
    """Equal rows with an inner product past half's range give equal outputs
    (to the roundings), also the last ones, which take the few-row form."""
    rows, n, k = 4100, 4096, 128
    assert adapter_of(rows, n, k, 1, 16) == (LARGE, 4)
    X = draw((1, k), dtype, 1).expand(rows, k).contiguous()
    W, A, B = draw((n, k), dtype, 2) * k ** -0.5, draw((1, 16, k), dtype, 3), draw((1, n, 16), dtype, 4) * 2.0 ** -12
    ids, scales = torch.zeros(rows, dtype=torch.int32, device="cuda"), torch.tensor([3e4], device="cuda")
    Y = call(X, W, ids, A, B, scales)
    want, bound = reference(X[:1], W, ids[:1], A, B, scales)
    assert float((X[:1].double() @ A[0].double().t()).abs().max()) * 3e4 > 65504
    close(Y, want, bound)


@pytest.mark.parametrize("rows, n, k, tile", FORMS)
def test_bfloat16_past_its_largest_number(rows, n, k, tile):
    """An inner product of 2^128 (1 - 2^-10), which is a float32 and would round to
    an infinity in bfloat16."""
    takes(rows, n, k, 2, 1, tile)
    zeros = lambda *s: torch.zeros(s, dtype=BF, device="cuda")  # noqa: E731
    X, W, A, B = zeros(rows, k), zeros(n, k), zeros(2, 1, k), zeros(2, n, 1)
    X[:, :2] = 2.0 ** 63
    A[1, 0, 0], A[1, 0, 1], B[:] = 2.0 ** 64 * (2 - 2.0 ** -7), 2.0 ** 64 * 1.5 * 2.0 ** -8, 2.0 ** -120
    ids, scales = torch.ones(rows, dtype=torch.int32, device="cuda"), torch.ones(2, device="cuda")
    close(call(X, W, ids, A, B, scales), *reference(X, W, ids, A, B, scales))


@pytest.mark.parametrize("dtype", [BF, HALF])
@pytest.mark.parametrize("rows, n, k, tile", FORMS + [(4096, 4096, 72, LARGE), (2304, 2048, 72, 1)])
def test_infinities_of_the_rows_own_adapter(dtype, rows, n, k, tile):
    """An infinity in B_a is one, with the sign of its product, in the column
    of every row of a (an h of either sign, from the first 64 ranks and the
    ones behind)."""
    takes(rows, n, k, 4, 72, tile)
    X, W, ids = draw((rows, k), dtype, 1), draw((n, k), dtype, 2) * k ** -0.5, ids_of(rows, 4)
    A, B = draw((4, 72, k), dtype, 3) * k ** -0.5, draw((4, n, 72), dtype, 4)
    scales = torch.tensor([1.0, 0.5, -2.0, 1.0], device="cuda")
    special = [(1, 5, 3, float("inf")), (2, 7, 0, float("-inf")), (2, n - 1, 71, float("inf")), (3, 0, 70, float("inf"))]
    want, _ = reference(X, W, ids, A, B, scales)
    sure = torch.ones_like(want, dtype=torch.bool)
    for a, c, r, v in special:
        B[a, c, r] = v
        rows_of = ids == a
        h = X[rows_of].double() @ A[a, r].double()
        want[rows_of, c] = torch.sign(h) * float(scales[a]) * v
        sure[rows_of, c] = h.abs() > k * 2.0 ** -22 * (X[rows_of].double().abs() @ A[a, r].double().abs())
    Y = call(X, W, ids, A, B, scales).double()
    finite = torch.isfinite(want)
    assert torch.equal(torch.isfinite(Y)[sure], finite[sure])
    assert torch.equal(Y[sure & ~finite], want[sure & ~finite])


@pytest.mark.parametrize("dtype", [BF, HALF])
@pytest.mark.parametrize("rank", [1, 5, 20, 70])
@pytest.mark.parametrize("rows, n, k, tile", FORMS)
def test_infinite_scales_and_activations(dtype, rank, rows, n, k, tile):
    """With positive operands every output that an infinity reaches is one: the
    ranks that pad an adapter add nothing."""
    takes(rows, n, k, 3, rank, tile)
    positive = lambda s, seed: draw(s, dtype, seed).abs().clamp(min=2.0 ** -6)  # noqa: E731
    X, W, A, B = positive((rows, k), 1), positive((n, k), 2), positive((3, rank, k), 3), positive((3, n, rank), 4)
    ids, scales = ids_of(rows, 3), torch.tensor([1.0, float("inf"), 0.0], device="cuda")
    scales[2] = 2.0 ** -6
    X *= 2.0 ** -3
    X[9, 0] = float("inf")
    Y = call(X, W, ids, A, B, scales)
    want = ids == 1
    want[9] = True
    assert torch.equal(torch.isposinf(Y), want[:, None].expand_as(Y)) and not torch.isnan(Y).any()
