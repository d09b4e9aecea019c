"""Calls that need no workspace are given none, eagerly and in a graph."""
import pytest
import torch

import gpu_util
import paper_2609_09095_amd as oz
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
