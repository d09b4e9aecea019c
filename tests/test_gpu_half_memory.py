"""Calls that need no workspace are given none, eagerly and in a graph."""
import pytest
import torch

import gpu_util
import paper_2609_09095_amd as oz
from test_gpu_grouped import draw
from test_gpu_orthogonalise import check, gradient

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def gpu():
    gpu_util.require_gpu()


@pytest.mark.parametrize("shape", [(2, 128, 128), (3, 40, 100), (1, 1, 1)])
def test_one_launch_in_a_graph_without_a_workspace(shape):
    G = gradient(shape, torch.float32)
    want = check(G)
    assert torch.equal(want, oz.ozaki25_orthogonalise(G, workspace=torch.empty(256, dtype=torch.uint8, device="cuda")))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        X = oz.ozaki25_orthogonalise(G)
    for seed in range(4):
        G.copy_(gradient(shape, torch.float32, seed + 7))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(X, oz.ozaki25_orthogonalise(G))


@pytest.mark.parametrize("rows, n", [(3, 64), (700, 520)])
def test_no_depth_and_no_adapters(rows, n):
    f = dict(dtype=torch.bfloat16, device="cuda")
    ids = torch.zeros(rows, dtype=torch.int32, device="cuda")
    E = torch.empty
    assert not oz.ozaki25_adapter_matmul(E(rows, 0, **f), E(n, 0, **f), ids, E(2, 24, 0, **f), E(2, n, 24, **f)).any()
    X, W = draw((rows, 64), torch.bfloat16, 0), draw((n, 64), torch.bfloat16, 1)
    none = oz.ozaki25_adapter_matmul(X, W, ids, E(0, 24, 64, **f), E(0, n, 24, **f))
    assert torch.equal(none, oz.ozaki25_adapter_matmul(X, W, ids - 1, E(2, 24, 64, **f).zero_(), E(2, n, 24, **f).zero_()))
