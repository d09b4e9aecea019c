"""The shared projection with adapters against the same sums in 64 bits.

Tolerance: with S = sum |x||w| and R = |s| sum |h||b|, h = sum x a, the FP32
sums err by at most (k + 2 rank + 8) 2^-23 (S + R') where R' bounds R with
sums of absolute values; h as two 16-bit numbers errs by 2^-16 |h| (bfloat16)
or 2^-22 |h| + 2^-24 (half, whose rest may be subnormal); then one rounding of
the result.
"""
import numpy as np
import pytest
import torch

import gpu_util
import paper_2609_09095_amd as oz
from test_gpu_grouped import TINY, UNIT, draw

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def gpu():
    gpu_util.require_gpu()


def reference(X, W, ids, A, B, scales):
    """(Y, bound) in 64 bits."""
    x, w = X.double(), W.double()
    Y, size = x @ w.t(), x.abs() @ w.abs().t()
    low = 2.0 ** -16 if X.dtype == torch.bfloat16 else 2.0 ** -22
    floor = 0.0 if X.dtype == torch.bfloat16 else 2.0 ** -24
    k, rank = X.shape[1], A.shape[1]
    err = torch.zeros_like(Y)
    for a in range(A.shape[0]):
        at = torch.nonzero(ids == a).flatten()
        if len(at) == 0:
            continue
        s = 1.0 if scales is None else float(scales[a])
        h, hs = x[at] @ A[a].double().t(), x[at].abs() @ A[a].double().abs().t()
        b = B[a].double()
        Y[at] += s * (h @ b.t())
        size[at] += abs(s) * (hs @ b.abs().t())
        err[at] += (abs(s) * low * hs + floor) @ b.abs().t()
    u = UNIT[X.dtype]
    return Y, ((k + 2 * rank + 8) * 2.0 ** -23 * size + err) * (1 + u) + u * Y.abs() + TINY[X.dtype]


def check(rows, n, k, adapters, rank, ids, dtype, scales=True, pad=0, shift=0, seed=0):
    gpu_util.log(f"adapter rows={rows} n={n} k={k} adapters={adapters} rank={rank} {dtype} pad={pad} shift={shift}")
    X, W = draw((rows, k), dtype, seed, pad, shift), draw((n, k), dtype, seed + 1, pad, shift)
    W *= max(k, 1) ** -0.5
    A, B = draw((adapters, rank, k), dtype, seed + 2, pad, shift), draw((adapters, n, rank), dtype, seed + 3, pad, shift)
    A *= max(k, 1) ** -0.5
    ids = torch.as_tensor(np.asarray(ids, dtype=np.int32)).cuda()
    s = torch.linspace(0.25, 2.0, adapters, device="cuda") if scales else None
    Y = oz.ozaki25_adapter_matmul(X, W, ids, A, B, s)
    torch.cuda.synchronize()
    want, bound = reference(X, W, ids, A, B, s)
    bad = ~((Y.double() - want).abs() <= bound)
    assert not bad.any(), (int(bad.sum()), float(((Y.double() - want).abs() / bound).max()))
    return X, W, ids, A, B, s, Y


def mixed(rows, adapters, seed=0):
    """Ids in any order, some naming no adapter."""
    return np.random.default_rng(seed).integers(-1, adapters, rows)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows", [1, 15, 17, 64, 100, 257, 700])
@pytest.mark.parametrize("n, k, rank", [(256, 512, 16), (264, 136, 8), (100, 77, 5), (1, 1, 1), (72, 1111, 24)])
def test_sizes(dtype, rows, n, k, rank):
    check(rows, n, k, 6, rank, mixed(rows, 6), dtype)


@pytest.mark.parametrize("rank", [1, 8, 16, 17, 32, 33, 48, 64, 65, 128, 130, 256])
@pytest.mark.parametrize("rows", [20, 300])
def test_ranks(rank, rows):
    check(rows, 136, 320, 3, rank, mixed(rows, 3), torch.bfloat16)


@pytest.mark.parametrize("rows", [64, 300])
def test_a_different_adapter_per_row(rows):
    check(rows, 128, 256, rows, 16, np.random.default_rng(1).permutation(rows), torch.bfloat16, scales=False)


def test_prompts_of_one_adapter_each():
    check(1100, 520, 1024, 4, 64, np.repeat([2, -1, 0, 3], [400, 100, 37, 563]), torch.bfloat16)


def test_ids_that_name_no_adapter():
    """Negative ids and ids past the last adapter: the projection alone."""
    for rows in (5, 300):
        X, W, ids, A, B, s, Y = check(rows, 64, 128, 2, 16, np.full(rows, -1), torch.bfloat16)
        for other in (-2 ** 31, 2, 2 ** 31 - 1):
            Y2 = oz.ozaki25_adapter_matmul(X, W, torch.full_like(ids, other), A, B, s)
            torch.cuda.synchronize()
            assert torch.equal(Y, Y2)


@pytest.mark.parametrize("pad, shift", [(8, 8), (3, 1), (0, 4), (1, 0)])
def test_pitches_and_alignment(pad, shift):
    for rows in (40, 300):
        check(rows, 136, 200, 3, 24, mixed(rows, 3), torch.float16, pad=pad, shift=shift)


def test_long_depth():
    for rows in (3, 300):
        check(rows, 40, 20000, 2, 16, mixed(rows, 2), torch.bfloat16)


@pytest.mark.parametrize("rows", [30, 300])
def test_infinities_stay_in_their_rows_and_adapters(rows):
    X, W, ids, A, B, s, Y = check(rows, 72, 136, 3, 16, np.arange(rows) % 4 - 1, torch.bfloat16)
    A[1, 3, 5] = float("nan")
    B[2, 7, 0] = float("inf")
    X[9, 0] = float("-inf")
    Y = oz.ozaki25_adapter_matmul(X, W, ids, A, B, s)
    torch.cuda.synchronize()
    want = torch.zeros_like(Y, dtype=torch.bool)
    want[ids == 1] = True
    want[ids == 2, 7] = True
    want[9] = True
    assert torch.equal(~torch.isfinite(Y), want)


def test_empty():
    f = dict(dtype=torch.bfloat16, device="cuda")
    ids = torch.zeros(4, dtype=torch.int32, device="cuda")
    E = torch.empty
    assert oz.ozaki25_adapter_matmul(E(0, 8, **f), E(8, 8, **f), ids[:0], E(2, 4, 8, **f), E(2, 8, 4, **f)).shape == (0, 8)
    assert oz.ozaki25_adapter_matmul(E(4, 8, **f), E(0, 8, **f), ids, E(2, 4, 8, **f), E(2, 0, 4, **f)).shape == (4, 0)
    assert not oz.ozaki25_adapter_matmul(E(4, 0, **f), E(8, 0, **f), ids, E(2, 4, 0, **f), E(2, 8, 4, **f)).any()
    X, W = draw((4, 16), torch.bfloat16, 0), draw((8, 16), torch.bfloat16, 1)
    want = oz.ozaki25_adapter_matmul(X, W, ids - 1, E(1, 4, 16, **f).zero_(), E(1, 8, 4, **f).zero_())
    assert torch.equal(want, oz.ozaki25_adapter_matmul(X, W, ids, E(0, 4, 16, **f), E(0, 8, 4, **f)))
    assert torch.equal(want, oz.ozaki25_adapter_matmul(X, W, ids, E(2, 0, 16, **f), E(2, 8, 0, **f)))


@pytest.mark.parametrize("rows", [20, 300])
def test_workspace_streams_and_repeats(rows):
    X, W, ids, A, B, s, want = check(rows, 264, 512, 4, 32, mixed(rows, 4), torch.bfloat16)
    need = oz.ozaki25_adapter_matmul_workspace_size(rows, 264, 512, 4, 32)
    room = torch.full((need,), 255, dtype=torch.uint8, device="cuda")  # NaN patterns: nothing stale is read
    other = torch.cuda.Stream()
    torch.cuda.synchronize()
    for kw in (dict(workspace=room), dict(stream=other), dict(stream=other.cuda_stream, workspace=room)):
        got = oz.ozaki25_adapter_matmul(X, W, ids, A, B, s, **kw)
        torch.cuda.synchronize()
        assert torch.equal(got, want)
    with pytest.raises(oz.Ozaki25Error):
        oz.ozaki25_adapter_matmul(X, W, ids, A, B, s, workspace=room[:need - 1])


@pytest.mark.parametrize("rows", [8, 300])
def test_in_a_graph(rows):
    X, W, ids, A, B, s, _ = check(rows, 136, 256, 4, 16, mixed(rows, 4), torch.bfloat16)
    room = torch.empty(oz.ozaki25_adapter_matmul_workspace_size(rows, 136, 256, 4, 16), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        Y = oz.ozaki25_adapter_matmul(X, W, ids, A, B, s, workspace=room)
    for seed in range(4):
        X.copy_(draw((rows, 256), torch.bfloat16, 20 + seed))
        ids.copy_(torch.from_numpy(mixed(rows, 4, seed).astype(np.int32)))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(Y, oz.ozaki25_adapter_matmul(X, W, ids, A, B, s))
