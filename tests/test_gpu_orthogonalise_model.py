"""The orthogonalisation against the model of its roundings (orth_model.py),
near enough to tell if its diagonals were rounded to half."""
import pytest
import torch

import gpu_util
import paper_2609_09095_amd as oz
from orth_model import bound, model
from test_gpu_orthogonalise import exact, gradient

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def gpu():
    gpu_util.require_gpu()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("shape", [(2, 128, 128), (2, 96, 128), (2, 128, 64), (1, 300, 520), (2, 515, 300), (2, 136, 1600),
                                   (1, 2048, 2048), (6, 2304, 2310)])
def test_the_roundings_are_the_stated_ones(shape, dtype):
    gpu_util.log(f"orthogonalise {shape} {dtype}")
    G = gradient(shape, dtype)
    X = oz.ozaki25_orthogonalise(G)
    torch.cuda.synchronize()
    scale = 32.0 if max(shape[1:]) <= 128 else 256.0
    for x, g in zip(X, G):
        want = model(g, scale_x=scale)
        off, most = (x.double() - want).norm(), bound(want, exact(g))
        assert off <= most, (float(off / want.norm()), float(most / want.norm()))
