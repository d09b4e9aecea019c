"""A layer of experts with an empty side gives zeros, or nothing to write, whatever
its weights are kept in; empty inputs of the other calls of the 8-bit path."""
import pytest

import gpu_util
import paper_2609_09095_amd as oz

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def gpu():
    gpu_util.require_gpu()


@pytest.mark.parametrize("gated", [True, False])
@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("tokens", [0, 3, 20])
@pytest.mark.parametrize("experts,width,inner,out,top", [(0, 200, 8, 136, 2), (3, 0, 8, 136, 2), (3, 200, 0, 136, 2), (3, 200, 8, 136, 0),
                                                         (3, 200, 8, 0, 2), (3, 0, 8, 0, 2), (3, 0, 0, 136, 2)])
def test_empty_sides(experts, width, inner, out, top, tokens, eight, gated):
    """The weights' values do not matter: they are NaN."""
    import torch

    def stack(rows, cols):
        W = torch.full((experts, rows, cols), float("nan"), dtype=torch.bfloat16, device="cuda")
        return oz.ozaki25_quantise(W, squares=True) if eight else (W, None)

    (up, us), (down, ds) = stack(inner, width), stack(out, inner)
    gate, gs = stack(inner, width) if gated else (None, None)
    X = torch.ones((tokens, width), dtype=torch.bfloat16, device="cuda")
    Y = torch.full((tokens, out), 3.0, dtype=torch.bfloat16, device="cuda")
    which = torch.zeros((tokens, top), dtype=torch.int32, device="cuda")
    got = oz.ozaki25_expert_layer(X, which, torch.ones((tokens, top), device="cuda"), up, down, gate=gate, up_scales=us,
                                  down_scales=ds, gate_scales=gs, Y=Y)
    assert got is Y and bool((Y == 0).all())


@pytest.mark.parametrize("rows,cols", [(0, 200), (200, 0), (0, 0)])
def test_empty_matrices(rows, cols):
    import torch
    X, w = torch.empty((rows, cols), dtype=torch.bfloat16, device="cuda"), torch.ones((cols,), dtype=torch.bfloat16, device="cuda")
    blocks = lambda n: -(-n // 128)  # noqa: E731
    for squares in (False, True):
        Q, s, QT, sT = oz.ozaki25_quantise(X, squares=squares, layout="both")
        assert Q.shape == (rows, cols) and QT.shape == (cols, rows)
        assert s.shape == ((blocks(rows), blocks(cols)) if squares else (blocks(cols), rows))
        assert sT.shape == ((blocks(cols), blocks(rows)) if squares else (blocks(rows), cols))
    for residual in (None, X):
        Q, s, *H = oz.ozaki25_rms_norm(X, w, residual=residual, quantised=True)
        assert Q.shape == (rows, cols) and s.shape == (blocks(cols), rows) and len(H) == (residual is not None)
        dX, dw = oz.ozaki25_rms_norm_backward(X, X, w, dH=residual)
        assert dX.shape == (rows, cols) and dw.shape == (cols,) and bool((dw == 0).all())
