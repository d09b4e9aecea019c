"""The 16-bit products do not record gradients, and say so where one is asked
for (on the CPU: before the tensors' device is checked)."""
import warnings

import pytest
import torch

import paper_2609_09095_amd as oz


def bf(*shape, grad=False):
    return torch.zeros(shape, dtype=torch.bfloat16, requires_grad=grad)


ENDS, IDS = torch.zeros(2, dtype=torch.int32), torch.zeros(4, dtype=torch.int32)
CALLS = {
    "grouped_matmul": (lambda g: (bf(4, 8, grad=g == 0), bf(2, 6, 8, grad=g == 1), ENDS), 2),
    "grouped_matmul_dx": (lambda g: (bf(4, 6, grad=g == 0), bf(2, 6, 8, grad=g == 1), ENDS), 2),
    "grouped_matmul_dw": (lambda g: (bf(4, 6, grad=g == 0), bf(4, 8, grad=g == 1), ENDS), 2),
    "adapter_matmul": (lambda g: (bf(4, 8, grad=g == 0), bf(6, 8, grad=g == 1), IDS, bf(3, 2, 8, grad=g == 2),
                                  bf(3, 6, 2, grad=g == 3), torch.zeros(3, requires_grad=g == 4)), 5),
    "orthogonalise": (lambda g: (bf(4, 8, grad=g == 0),), 1),
}


@pytest.mark.parametrize("name", CALLS)
def test_a_gradient_that_would_be_lost_is_told(name):
    f, (args, inputs) = getattr(oz, f"ozaki25_{name}"), CALLS[name]
    for g in range(inputs):
        with pytest.warns(UserWarning, match="does not record"), pytest.raises(ValueError, match="CUDA tensor"):
            f(*args(g))
    with warnings.catch_warnings():
        warnings.simplefilter("error")
        with pytest.raises(ValueError, match="CUDA tensor"):
            f(*args(-1))
        with torch.no_grad(), pytest.raises(ValueError, match="CUDA tensor"):
            f(*args(0))


def test_the_warning_points_at_the_call():
    with pytest.warns(UserWarning) as told, pytest.raises(ValueError):
        oz.ozaki25_orthogonalise(bf(4, 8, grad=True))
    assert told[0].filename == __file__
