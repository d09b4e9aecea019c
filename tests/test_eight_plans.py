"""The plan of an 8-bit product is that of the form which runs, wherever its operands
lie, and the stated workspace holds it."""
import ctypes

import pytest

import eight_routes
import paper_2609_09095_amd as oz

FEW16, FEW32, FEW48, SMALL, MIDDLE, LARGE = range(6)
SIZES = [1, 4, 5, 8, 9, 15, 16, 17, 32, 48, 49, 64, 65, 128, 300, 1000, 2944, 2945, 3200, 3201, 4095, 4096, 4097, 5120, 5121, 8191, 70000, 1 << 22]


@pytest.fixture(scope="module")
def L():
    return eight_routes.plans()


@pytest.fixture(scope="module", autouse=True)
def built_library():
    import os
    if not os.path.exists(oz.library_path()):
        from paper_2609_09095_amd import build
        build.build()
    oz.lib()


def test_words_and_dma(L):
    for c, words, dma in (((0, 16, 16, 32), 1, 1), ((16, 16, 8, 32), 1, 0), ((4, 20, 12, 4), 1, 0), ((2, 16, 0, 16), 0, 0),
                          ((0, 17, 0, 16), 0, 0), ((0, 16, 3, 16), 0, 0), ((0, 16, 0, 30), 0, 0), ((0, 1 << 22, 0, 16), 1, 0),
                          ((0, 16, 0, 1 << 22), 1, 0), ((0, (1 << 22) - 16, 0, 16), 1, 1), ((0, 1 << 32, 0, 16), 1, 0)):
        assert (L.plan_words(*c), L.plan_dma(*c)) == (words, dma), c


def test_forms_on_the_measured_side(L):
    for c, want in (((17, 64, 2000, 1), (FEW32, 1)), ((32, 4096, 4092, 1), (FEW32, 1)), ((48, 4096, 3001, 1), (FEW48, 1)),
                    ((17, 64, 4095, 0), (SMALL, 4)), ((32, 256, 4095, 0), (SMALL, 4)), ((48, 4096, 2047, 0), (SMALL, 1)),
                    ((16, 4096, 4095, 0), (SMALL, 4)), ((16, 4096, 3001, 0), (FEW16, 1)), ((1, 4096, 2047, 0), (FEW16, 1)),
                    ((8, 4096, 3843, 0), (FEW16, 1)), ((8, 4096, 4225, 0), (SMALL, 4)), ((1, 4096, 5001, 0), (FEW16, 1)),
                    ((1, 4096, 8191, 0), (SMALL, 8)), ((16, 8192, 8192, 1), (FEW16, 1)), ((49, 4096, 4095, 0), (SMALL, 4)), ((49, 4096, 4095, 1), (SMALL, 4))):
        assert (L.plan_form(*c), L.plan_split(*c)) == want, c


def test_every_plan_holds(L):
    """Parts of at least 8 blocks, only of forms that split; at least as many as the same
    tiles have with one row more; the workspace holds either plan's parts."""
    size = oz.lib().ozaki25_scaled_matmul_workspace_size
    for rows in SIZES + [1 << 30]:
        for n in SIZES:
            for k in SIZES:
                rooms = []
                for words in (0, 1):
                    form, split = L.plan_form(rows, n, k, words), L.plan_split(rows, n, k, words)
                    assert 1 <= split <= 8 and (split == 1 or (form in (SMALL, MIDDLE) and -(-k // 128) >= 8 * split))
                    assert form not in (FEW16, FEW32, FEW48) or rows <= {FEW16: 16, FEW32: 32, FEW48: 48}[form]
                    if form == SMALL and rows < 49 and L.plan_form(49, n, k, words) == SMALL:
                        assert split == L.plan_split(49, n, k, words)
                    rooms.append(0 if split == 1 else split * rows * (-(-n // 4) * 4) * 4)
                    assert L.plan_room(rows, n, k, words) == rooms[-1]
                assert size(rows, n, k) == -(-max(rooms) // 256) * 256


def test_a_workspace_too_small_for_the_form_that_runs():
    """32 x 256 x 4095 at odd places: parts, which a byte less does not hold."""
    p = lambda i, off=0: ctypes.c_void_p((i << 32) + off)  # noqa: E731
    need = oz.ozaki25_scaled_matmul_workspace_size(32, 256, 4095)
    assert need == 4 * 32 * 256 * 4
    for off, lda in ((1, 4096), (0, 4095)):
        assert oz.lib().ozaki25_scaled_matmul(32, 256, 4095, p(1, off), lda, p(2), 32, p(3), 4096, p(4), 32, 1, p(5), 256, oz.BF16,
                                              p(6), need - 1, None) == oz.ERR_WORKSPACE
