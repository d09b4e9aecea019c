"""The grouped products and both gradients against the same products in 64
bits.

Tolerance, from the arithmetic: products of 16-bit operands are exact in FP32,
their sum over d terms errs by at most d 2^-24 S with S = sum |a||b| (each of
at most d additions rounds once, to nearest or toward zero, a partial sum of
at most S: d 2^-23 S in the worst case), and the result is rounded once more:
u |c| with u = 2^-8 (bfloat16), 2^-11 (half), 2^-24 (float32).
"""
import numpy as np
import pytest
import torch

import gpu_util
import paper_2609_09095_amd as oz

pytestmark = pytest.mark.gpu

UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
TINY = {torch.bfloat16: 2.0 ** -126, torch.float16: 2.0 ** -24, torch.float32: 2.0 ** -126}


@pytest.fixture(scope="module", autouse=True)
def gpu():
    gpu_util.require_gpu()


def draw(shape, dtype, seed, pad=0, shift=0):
    """Normal values in a wider matrix, its rows `pad` elements longer and its
    first element `shift` elements past a fresh allocation."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    pitch = shape[-1] + pad
    count = int(np.prod(shape[:-1])) * pitch + shift
    flat = torch.full((count,), float("nan"), dtype=dtype, device="cuda")
    view = flat[shift:].view(*shape[:-1], pitch)[..., :shape[-1]]
    view.normal_(0.0, 1.0, generator=gen)
    return view


def spans(ends, rows):
    out, last = [], 0
    for e in ends:
        e = min(max(e, last), rows)
        out.append((last, e))
        last = e
    return out, last


def close(got, want, size, depth):
    """|got - want| within the bound; size: sum |a||b|."""
    u = UNIT[got.dtype]
    bound = depth * 2.0 ** -23 * size * (1 + u) + u * want.abs() + TINY[got.dtype]
    d = (got.double() - want).abs()
    bad = ~(d <= bound)
    assert not bad.any(), (int(bad.sum()), float((d / bound).max()))


def check_all(rows, n, k, sizes, dtype, pad=0, shift=0, seed=0):
    ends = np.cumsum(sizes).tolist()
    gpu_util.log(f"grouped rows={rows} n={n} k={k} ends={ends[:8]} {dtype} pad={pad} shift={shift}")
    groups = len(sizes)
    X, dY = draw((rows, k), dtype, seed, pad, shift), draw((rows, n), dtype, seed + 1, pad, shift)
    W = draw((groups, n, k), dtype, seed + 2, pad, shift)
    E = torch.tensor(ends, dtype=torch.int32, device="cuda")
    Y = oz.ozaki25_grouped_matmul(X, W, E)
    dX = oz.ozaki25_grouped_matmul_dx(dY, W, E)
    dWs = [oz.ozaki25_grouped_matmul_dw(dY, X, E, out_dtype=t) for t in (dtype, torch.float32)]
    torch.cuda.synchronize()
    parts, last = spans(ends, rows)
    assert torch.count_nonzero(Y[last:]) == 0 and torch.count_nonzero(dX[last:]) == 0
    for g, (i, j) in enumerate(parts):
        x, dy, w = X[i:j].double(), dY[i:j].double(), W[g].double()
        close(Y[i:j], x @ w.t(), x.abs() @ w.abs().t(), k)
        close(dX[i:j], dy @ w, dy.abs() @ w.abs(), n)
        for dW in dWs:
            close(dW[g], dy.t() @ x, dy.abs().t() @ x.abs(), max(j - i, 1))


# a row tile's edges, one row, no rows, groups that end inside a tile
SIZES = [
    [1], [0, 1, 0], [255, 1, 256, 257], [3, 0, 70, 129, 0, 500], [64] * 5, [1] * 70, [0] * 64 + [5, 0, 130],
]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: f"{len(s)}groups_{sum(s)}rows")
@pytest.mark.parametrize("n, k", [(8, 8), (264, 136), (128, 512), (1, 1), (7, 3), (133, 65), (320, 257)])
def test_sizes(dtype, sizes, n, k):
    check_all(sum(sizes), n, k, sizes, dtype)


@pytest.mark.parametrize("pad, shift", [(8, 0), (8, 8), (0, 4), (3, 1), (1, 0), (0, 1)])
def test_pitches_and_alignment(pad, shift):
    check_all(300, 264, 200, [100, 0, 150, 50], torch.bfloat16, pad, shift)
    check_all(300, 77, 111, [100, 0, 150, 50], torch.float16, pad, shift)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_many_rows_and_columns(dtype):
    check_all(3000, 1024, 512, [700, 0, 1800, 33, 467], dtype)


def test_long_depth():
    check_all(40, 64, 70000, [17, 23], torch.bfloat16)
    check_all(70001, 24, 40, [70000, 1], torch.bfloat16)


def test_rows_past_the_last_end():
    check_all(600, 72, 80, [10, 0, 300], torch.bfloat16)
    check_all(600, 71, 81, [10, 0, 300], torch.float16)


@pytest.mark.parametrize("n", [64, 65])
def test_ends_out_of_order_or_range(n):
    """An end below the one before it is an empty group, one past the rows
    stops there."""
    rows, k = 500, 64
    X, W = draw((rows, k), torch.bfloat16, 3), draw((5, n, k), torch.bfloat16, 4)
    ends = [200, 100, -7, 1 << 30, 40]
    E = torch.tensor(ends, dtype=torch.int32, device="cuda")
    Y, dW = oz.ozaki25_grouped_matmul(X, W, E), oz.ozaki25_grouped_matmul_dw(X, X, E)
    torch.cuda.synchronize()
    parts, last = spans(ends, rows)
    assert parts == [(0, 200), (200, 200), (200, 200), (200, 500), (500, 500)] and last == rows
    for g, (i, j) in enumerate(parts):
        x, w = X[i:j].double(), W[g].double()
        close(Y[i:j], x @ w.t(), x.abs() @ w.abs().t(), k)
        close(dW[g], x.t() @ x, x.abs().t() @ x.abs(), rows)


@pytest.mark.parametrize("n, k", [(72, 200), (71, 201)])
def test_infinities_stay_in_their_rows_and_groups(n, k):
    """A NaN or infinity reaches the outputs that read it and no other: not the
    neighbouring group through a tile's edge, nor past the end of the depth."""
    sizes = [70, 58, 72]
    rows = sum(sizes)
    X, W, dY = (draw(s, torch.bfloat16, i) for i, s in enumerate([(rows, k), (3, n, k), (rows, n)]))
    X[75, k - 1] = float("inf")   # group 1
    dY[3, 0] = float("nan")       # group 0
    W[2, 5, 0] = float("-inf")
    E = torch.tensor(np.cumsum(sizes).tolist(), dtype=torch.int32, device="cuda")
    Y = oz.ozaki25_grouped_matmul(X, W, E)
    dX = oz.ozaki25_grouped_matmul_dx(dY, W, E)
    dW = oz.ozaki25_grouped_matmul_dw(dY, X, E)
    torch.cuda.synchronize()
    bad = torch.zeros_like(Y, dtype=torch.bool)
    bad[75] = True
    bad[128:, 5] = True
    assert torch.equal(~torch.isfinite(Y), bad)
    bad = torch.zeros_like(dX, dtype=torch.bool)
    bad[3] = True
    bad[128:, 0] = True
    assert torch.equal(~torch.isfinite(dX), bad)
    bad = torch.zeros_like(dW, dtype=torch.bool)
    bad[0, 0] = True
    bad[1, :, k - 1] = True
    assert torch.equal(~torch.isfinite(dW), bad)


def test_shared_weights_and_output_views():
    """Weights expanded over the groups (stride 0), outputs inside wider
    buffers whose other elements keep their values."""
    rows, n, k = 130, 48, 64
    X, W1 = draw((rows, k), torch.bfloat16, 1), draw((1, n, k), torch.bfloat16, 2)
    E = torch.tensor([30, 100, 130], dtype=torch.int32, device="cuda")
    for pad in (3, 16):
        wide = torch.full((rows, n + pad), 7.0, dtype=torch.bfloat16, device="cuda")
        Y = oz.ozaki25_grouped_matmul(X, W1.expand(3, n, k), E, Y=wide[:, :n])
        torch.cuda.synchronize()
        close(Y, X.double() @ W1[0].double().t(), X.double().abs() @ W1[0].double().abs().t(), k)
        assert bool((wide[:, n:] == 7.0).all())
        wide = torch.full((3, n + 1, k + pad), 7.0, device="cuda")
        dW = oz.ozaki25_grouped_matmul_dw(Y, X, E, dW=wide[:, :n, :k])
        torch.cuda.synchronize()
        y = Y.double()
        close(dW[1], y[30:100].t() @ X[30:100].double(), y[30:100].abs().t() @ X[30:100].double().abs(), 70)
        assert bool((wide[:, n:] == 7.0).all()) and bool((wide[:, :, k:] == 7.0).all())


def test_empty():
    f = dict(dtype=torch.bfloat16, device="cuda")
    E = torch.tensor([4, 4], dtype=torch.int32, device="cuda")
    assert oz.ozaki25_grouped_matmul(torch.empty(0, 8, **f), torch.empty(2, 8, 8, **f), E).shape == (0, 8)
    assert oz.ozaki25_grouped_matmul(torch.empty(4, 8, **f), torch.empty(2, 0, 8, **f), E).shape == (4, 0)
    assert not oz.ozaki25_grouped_matmul(torch.empty(4, 0, **f), torch.empty(2, 8, 0, **f), E).any()
    assert not oz.ozaki25_grouped_matmul(torch.empty(4, 8, **f).fill_(1), torch.empty(0, 8, 8, **f), E[:0]).any()
    assert not oz.ozaki25_grouped_matmul_dw(torch.empty(0, 8, **f), torch.empty(0, 8, **f), E).any()


def test_gradients_against_differences():
    """<dY, Y(X + h D) - Y(X - h D)> / 2h equals <dX, D>, and for W <dW, D>:
    with integers of few bits every product and sum is exact."""
    gen = torch.Generator(device="cuda").manual_seed(5)

    def ints(*shape):
        return torch.randint(-3, 4, shape, device="cuda", generator=gen).to(torch.bfloat16)

    rows, n, k = 90, 40, 56
    E = torch.tensor([20, 20, 77], dtype=torch.int32, device="cuda")
    X, W, dY, DX, DW = ints(rows, k), ints(3, n, k), ints(rows, n), ints(rows, k), ints(3, n, k)

    def loss(X, W):  # float16 holds the outputs exactly: integers below 2048
        Y = oz.ozaki25_grouped_matmul(X.half(), W.half(), E)
        return float((Y.double() * dY.double()).sum())

    dX = oz.ozaki25_grouped_matmul_dx(dY.half(), W.half(), E).double()
    dW = oz.ozaki25_grouped_matmul_dw(dY, X, E, out_dtype=torch.float32).double()
    assert (loss(X + DX, W) - loss(X - DX, W)) / 2 == float((dX * DX.double()).sum())
    assert (loss(X, W + DW) - loss(X, W - DW)) / 2 == float((dW * DW.double()).sum())


def test_repeats_bit_for_bit_and_on_another_stream():
    X, W = draw((700, 512), torch.bfloat16, 1), draw((4, 264, 512), torch.bfloat16, 2)
    E = torch.tensor([100, 350, 360, 700], dtype=torch.int32, device="cuda")
    V = W.transpose(1, 2).contiguous()
    want = [oz.ozaki25_grouped_matmul(X, W, E), oz.ozaki25_grouped_matmul_dx(X, V, E),
            oz.ozaki25_grouped_matmul_dw(X, X, E)]
    torch.cuda.synchronize()
    other = torch.cuda.Stream()
    for stream in (None, other, other.cuda_stream):
        got = [oz.ozaki25_grouped_matmul(X, W, E, stream=stream),
               oz.ozaki25_grouped_matmul_dx(X, V, E, stream=stream),
               oz.ozaki25_grouped_matmul_dw(X, X, E, stream=stream)]
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b)


def test_in_a_graph():
    """Captured once, replayed with other inputs and group ends in the same
    buffers; every replay equals the eager call."""
    X, W = draw((300, 256), torch.bfloat16, 1), draw((3, 136, 256), torch.bfloat16, 2)
    E = torch.tensor([100, 200, 300], dtype=torch.int32, device="cuda")
    oz.ozaki25_grouped_matmul(X, W, E)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        Y = oz.ozaki25_grouped_matmul(X, W, E)
        dX = oz.ozaki25_grouped_matmul_dx(Y, W, E)
        dW = oz.ozaki25_grouped_matmul_dw(Y, X, E)
    for seed, ends in enumerate([(100, 200, 300), (0, 17, 300), (300, 300, 300), (5, 6, 7)]):
        X.copy_(draw((300, 256), torch.bfloat16, 10 + seed))
        E.copy_(torch.tensor(ends, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        y = oz.ozaki25_grouped_matmul(X, W, E)
        assert torch.equal(Y, y) and torch.equal(dX, oz.ozaki25_grouped_matmul_dx(y, W, E))
        assert torch.equal(dW, oz.ozaki25_grouped_matmul_dw(y, X, E))
