"""The 16-bit products ask for the memory that they use (on the CPU)."""
import pytest

import paper_2609_09095_amd as oz


@pytest.fixture(scope="module", autouse=True)
def built_library():
    import os
    if not os.path.exists(oz.library_path()):
        from paper_2609_09095_amd import build
        build.build()
    oz.lib()


@pytest.mark.parametrize("count, m, n", [(1, 1, 1), (32, 128, 128), (65535, 128, 128), (64, 128, 7), (3, 5, 128)])
def test_matrices_of_one_launch_need_no_room(count, m, n):
    """The least that a workspace is: one unit of its alignment."""
    assert oz.ozaki25_orthogonalise_workspace_size(count, m, n) == 256


@pytest.mark.parametrize("m, n", [(129, 1), (1, 129), (128, 136), (200, 128)])
def test_larger_ones_need_it(m, n):
    assert oz.ozaki25_orthogonalise_workspace_size(4, m, n) > 4 * m * n * 8
