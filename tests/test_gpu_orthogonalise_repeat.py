"""Equal calls give equal bits: the last step's tiles read X through LDS in
two halves, the second one into the first one's place."""
import pytest
import torch

import gpu_util
import paper_2609_09095_amd as oz
from half_routes import LARGE, MIDDLE, SMALL, rules
from test_gpu_orthogonalise import check, gradient

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def gpu():
    gpu_util.require_gpu()


@pytest.mark.parametrize("count, m, n, tile", [(2, 3000, 4100, LARGE), (2, 4100, 3000, LARGE), (6, 2304, 2310, LARGE),
                                               (2, 4096, 4096, LARGE), (3, 1400, 1500, MIDDLE), (3, 1537, 515, SMALL)])
@pytest.mark.parametrize("steps", [1, 2])
def test_repeats(count, m, n, tile, steps):
    up = lambda b: count * -(-m // b) * -(-n // b)  # noqa: E731
    assert rules().rule_tile_of(up(128), up(256)) == tile
    G = gradient((count, m, n), torch.float32)
    want = check(G, steps=steps)
    for _ in range(40):
        assert torch.equal(oz.ozaki25_orthogonalise(G, steps=steps), want)
