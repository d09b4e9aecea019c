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


@pytest.mark.parametrize("rows, n", [(1, 64), (64, 4096), (700, 520), (4100, 4096)])
def test_adapters_that_nothing_reaches_need_no_room(rows, n):
    size = oz.ozaki25_adapter_matmul_workspace_size
    assert size(rows, n, 0, 8, 64) == size(rows, n, 0, 8, 0) == size(rows, n, 0, 0, 0)
    assert size(rows, n, 1024, 0, 64) == size(rows, n, 1024, 8, 0) < size(rows, n, 1024, 8, 64)
