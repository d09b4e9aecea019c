"""The rules by which the 8-bit path chooses its kernels, on the CPU: on the faster
side at sizes that were measured both ways, and within their limits over all sizes."""
import ctypes
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FEW16, FEW32, FEW48, SMALL, MIDDLE, LARGE = range(6)
ONE, NARROW, WIDE, ROWS, MANY = range(5)


@pytest.fixture(scope="module")
def L(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("rules") / "librules.so")
    subprocess.run(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", "-Wall", "-Werror",
                    "-I" + os.path.join(ROOT, "paper_2609_09095_amd", "csrc"), "-o", out,
                    os.path.join(ROOT, "tests", "host", "eight_rules.cpp")], check=True)
    lib = ctypes.CDLL(out)
    i64, i32 = ctypes.c_int64, ctypes.c_int
    for name, args, res in (("norm_lanes", [i64], i32), ("norm_chunks", [i64], i32), ("norm_threads", [i64], i32),
                            ("norm_blocks", [i64] * 2, i64), ("norm_parts", [i64] * 2, i64), ("scaled_form", [i64] * 3, i32),
                            ("scaled_split", [i64] * 3, i32), ("scaled_tall", [i64] * 2, i32), ("scaled_room", [i64] * 3, i64), ("together", [i64] * 2, i32), ("share_rows", [i64] * 3, i32),
                            ("hidden", [i64, i64, i64, i32, i32], i32)):
        f = getattr(lib, "rule_" + name)
        f.argtypes, f.restype = args, res
    return lib


def test_norms_hold_every_row(L):
    """Lanes of 8 columns a chunk cover the width and no chunk is wholly idle; a block
    is whole rows; blocks beyond the rows are not launched."""
    for width in list(range(1, 2100)) + list(range(2100, 32769, 61)) + [32768]:
        lanes, chunks, threads = L.rule_norm_lanes(width), L.rule_norm_chunks(width), L.rule_norm_threads(width)
        assert lanes * chunks * 8 >= width and lanes * (chunks - 1) * 8 < width or (lanes, chunks) == (1024, 4)
        assert threads % lanes == 0 and threads <= 1024 and lanes % 16 == 0 and (lanes <= 64 or threads == lanes)
        for rows in (1, 7, 4000, 1 << 30):
            blocks, parts = L.rule_norm_blocks(rows, width), L.rule_norm_parts(rows, width)
            per = threads // lanes
            assert 1 <= parts <= blocks <= min(-(-rows // per), 256 * max(1, 2048 // threads))


def test_scaled_forms_on_the_measured_side(L):
    for c, want in (((1, 4096, 4096), (FEW16, 1)), ((16, 8192, 8192), (FEW16, 1)), ((17, 4096, 4096), (FEW32, 1)),
                    ((33, 4096, 4096), (FEW48, 1)), ((32, 8192, 8192), (SMALL, 6)), ((64, 1024, 8192), (SMALL, 8)),
                    ((64, 64, 8192), (SMALL, 8)), ((65, 4096, 4096), (SMALL, 2)), ((300, 4096, 4096), (SMALL, 1)),
                    ((512, 4096, 4096), (SMALL, 1)), ((333, 1000, 1111), (SMALL, 1)), ((512, 512, 8192), (SMALL, 8)),
                    ((285, 128, 7355), (SMALL, 7)), ((1024, 1024, 16384), (MIDDLE, 8)), ((2048, 2048, 2048), (MIDDLE, 1)),
                    ((2048, 4096, 8192), (MIDDLE, 1)), ((16384, 4096, 4096), (LARGE, 1)), ((4096, 4096, 4096), (LARGE, 1))):
        assert (L.rule_scaled_form(*c), L.rule_scaled_split(*c)) == want, c


def test_parts_have_depths_and_room(L):
    """Every part of a split depth has at least 8 blocks of 128; the room is that of
    the parts' sums."""
    sizes = [1, 15, 16, 17, 63, 64, 65, 128, 129, 300, 1000, 4096, 70000, 1 << 22, 1 << 30]
    for rows in sizes:
        for n in sizes[:-1]:
            for k in sizes[:-1]:
                split, form = L.rule_scaled_split(rows, n, k), L.rule_scaled_form(rows, n, k)
                assert 1 <= split <= 8 and (split == 1 or (form in (SMALL, MIDDLE) and -(-k // 128) >= 8 * split))
                assert L.rule_scaled_room(rows, n, k) == (0 if split == 1 else split * rows * (-(-n // 4) * 4) * 4)
                assert L.rule_scaled_room(rows, n, k) < 1 << 30


def test_tall_tiles_on_the_measured_side(L):
    """256 x 128 where the card is full of them; such a product's depth is whole."""
    for c, want in (((2048, 4096), 1), ((4096, 4096), 1), ((3300, 2050), 1), ((2048, 2048), 0), ((1024, 4096), 0),
                    ((2049, 2050), 0)):
        assert L.rule_scaled_tall(*c) == want, c
        for k in (1, 4096, 1 << 22):
            assert not want or (L.rule_scaled_form(*c, k) in (MIDDLE, LARGE) and L.rule_scaled_split(*c, k) == 1)


def test_layers_on_the_measured_side(L):
    for c, want in (((1, 2), 1), ((4, 2), 1), ((16, 1), 1), ((1, 17), 0), ((16, 4), 0), ((64, 4), 0)):
        assert L.rule_together(*c) == want, c
    for c, want in (((2, 2, 1024, 1, 0), ONE), ((8, 8, 2048, 1, 0), NARROW), ((64, 8, 1024, 1, 1), WIDE),
                    ((256, 64, 1024, 1, 1), WIDE), ((256, 64, 1024, 1, 0), WIDE), ((128, 8, 1024, 1, 0), ROWS),
                    ((1, 1, 1, 0, 0), ONE), ((40, 20, 500, 1, 0), NARROW), ((128, 64, 900, 0, 0), WIDE),
                    ((260, 20, 500, 0, 1), ROWS), ((512, 16, 1024, 1, 0), MANY), ((256, 8, 2048, 1, 1), MANY),
                    ((800, 64, 270, 1, 0), MANY), ((400, 16, 2050, 0, 1), MANY), ((480, 16, 1030, 0, 1), ROWS)):
        assert L.rule_hidden(*c) == want, c
    for c, want in (((512, 16, 2048), 1), ((256, 8, 2048), 1), ((128, 8, 4096), 1), ((800, 64, 250), 1), ((64, 2, 2048), 0),
                    ((256, 64, 2048), 0)):
        assert L.rule_share_rows(*c) == want, c
