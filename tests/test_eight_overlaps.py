"""What counts as overlapping in the 8-bit path: all from a matrix's first to its last
element, slices of the same rows among it; the sum's and the gradient's own memory is
their whole matrix."""
import ctypes

import pytest

import paper_2609_09095_amd as oz


@pytest.fixture(scope="module", autouse=True)
def built_library():
    import os
    if not os.path.exists(oz.library_path()):
        from paper_2609_09095_amd import build
        build.build()
    oz.lib()


def p(i, off=0):
    return ctypes.c_void_p((i << 32) + off)


def test_slices_of_the_same_rows():
    norm, grad, mm = oz.lib().ozaki25_rms_norm, oz.lib().ozaki25_rms_norm_backward, oz.lib().ozaki25_scaled_matmul
    bad = oz.ERR_INVALID_VALUE
    # 8 rows of 100 beside each other in rows of 200 elements of 2 bytes: Y beside X, H = X beside the residual
    assert norm(8, 100, p(1), 200, None, 1, None, oz.BF16, 1e-6, None, 1, p(1, 200), 200, None, 1, None) == bad
    assert norm(8, 100, p(1), 200, p(1, 200), 200, None, oz.BF16, 1e-6, p(1), 200, p(2), 100, None, 1, None) == bad
    # dX over dY's memory but beside H
    assert grad(8, 100, p(1), 200, p(1, 200), 200, None, None, 1, oz.BF16, 1e-6, p(1), 200, p(2), p(3), 1 << 20, None) == bad
    assert mm(8, 100, 100, p(1), 300, p(2), 8, p(3), 100, p(4), 1, 1, p(1, 100), 150, oz.BF16, None, 0, None) == bad
