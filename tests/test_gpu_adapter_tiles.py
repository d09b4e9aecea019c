"""The whole-tile form of the shared projection with adapters, at sizes that
the rules send there (asserted), behind either product X A^T: what
`test_gpu_adapter.py` asks of the operator's smaller calls."""
import numpy as np
import pytest
import torch

import gpu_util
import paper_2609_09095_amd as oz
from half_routes import adapter_of
from test_gpu_adapter import check, mixed
from test_gpu_grouped import draw

pytestmark = pytest.mark.gpu

BF, HALF = torch.bfloat16, torch.float16
# below and above 1024 rows, from which on X A^T runs in tiles of its own
ROWS = [700, 1090]


@pytest.fixture(scope="module", autouse=True)
def gpu():
    gpu_util.require_gpu()


def tiles(rows, n, k, adapters, rank, ids, dtype, **kw):
    tile, served = adapter_of(rows, n, k, adapters, rank)
    assert tile is not None and served == 0
    return check(rows, n, k, adapters, rank, ids, dtype, **kw)


@pytest.mark.parametrize("rows", ROWS)
@pytest.mark.parametrize("rank", [1, 8, 16, 17, 32, 33, 48, 64, 65, 128, 130, 256])
def test_ranks(rank, rows):
    for dtype in (BF, HALF):
        tiles(rows, 136, 320, 3, rank, mixed(rows, 3), dtype)


@pytest.mark.parametrize("dtype", [BF, HALF])
@pytest.mark.parametrize("rows, n, k", [(513, 136, 256), (520, 77, 1), (641, 1, 1000), (1024, 1, 8), (1025, 264, 77)])
def test_sizes(dtype, rows, n, k):
    tiles(rows, n, k, 6, 20, mixed(rows, 6), dtype)


@pytest.mark.parametrize("rows", ROWS)
def test_a_different_adapter_per_row(rows):
    tiles(rows, 128, 256, rows, 16, np.random.default_rng(1).permutation(rows), BF, scales=False)


@pytest.mark.parametrize("rows", ROWS)
def test_ids_that_name_no_adapter(rows):
    X, W, ids, A, B, s, Y = tiles(rows, 64, 128, 2, 16, np.full(rows, -1), BF)
    for other in (-2 ** 31, 2, 2 ** 31 - 1):
        Y2 = oz.ozaki25_adapter_matmul(X, W, torch.full_like(ids, other), A, B, s)
        torch.cuda.synchronize()
        assert torch.equal(Y, Y2)


@pytest.mark.parametrize("rows", ROWS)
@pytest.mark.parametrize("pad, shift", [(8, 8), (3, 1), (0, 4), (1, 0)])
def test_pitches_and_alignment(pad, shift, rows):
    tiles(rows, 136, 200, 3, 24, mixed(rows, 3), HALF, pad=pad, shift=shift)


@pytest.mark.parametrize("rows", ROWS)
def test_long_depth(rows):
    tiles(rows, 40, 20000, 2, 16, mixed(rows, 2), BF)


@pytest.mark.parametrize("rows", ROWS)
@pytest.mark.parametrize("dtype", [BF, HALF])
def test_infinities_stay_in_their_rows_and_adapters(rows, dtype):
    X, W, ids, A, B, s, Y = tiles(rows, 72, 136, 3, 16, np.arange(rows) % 4 - 1, dtype)
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


@pytest.mark.parametrize("rows", ROWS)
def test_workspace_streams_and_repeats(rows):
    X, W, ids, A, B, s, want = tiles(rows, 264, 512, 4, 32, mixed(rows, 4), HALF)
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


@pytest.mark.parametrize("rows", ROWS)
def test_in_a_graph(rows):
    X, W, ids, A, B, s, _ = tiles(rows, 136, 256, 4, 16, mixed(rows, 4), HALF)
    room = torch.empty(oz.ozaki25_adapter_matmul_workspace_size(rows, 136, 256, 4, 16), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        Y = oz.ozaki25_adapter_matmul(X, W, ids, A, B, s, workspace=room)
    for seed in range(4):
        X.copy_(draw((rows, 256), HALF, 20 + seed))
        ids.copy_(torch.from_numpy(mixed(rows, 4, seed).astype(np.int32)))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(Y, oz.ozaki25_adapter_matmul(X, W, ids, A, B, s))
