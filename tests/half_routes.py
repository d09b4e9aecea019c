"""Which form a 16-bit product takes: the library's own rules
(paper_2609_09095_amd/csrc/half_rules.hpp), compiled with g++ on first use, so
that a test of one form can assert that its sizes still reach it."""
from __future__ import annotations

import ctypes
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2609_09095_amd", "csrc")
_HOST = os.path.join(ROOT, "tests", "host")
_SRC = os.path.join(_HOST, "half_rules.cpp")
_HDR = os.path.join(CSRC, "half_rules.hpp")
_LIB = os.path.join(_HOST, "libhalfrules.so")
_lib = None

SMALL, MIDDLE, LARGE = range(3)
FEW16, FEW32, FEW64X32, FEW64X64 = range(4)


def rules():
    global _lib
    if _lib is None:
        newest = max(os.path.getmtime(_SRC), os.path.getmtime(_HDR))
        if not os.path.exists(_LIB) or os.path.getmtime(_LIB) < newest:
            tmp = _LIB + ".tmp%d" % os.getpid()
            subprocess.check_call(["g++", "-O2", "-std=c++20", "-shared", "-fPIC", f"-I{CSRC}", "-o", tmp, _SRC])
            os.replace(tmp, _LIB)
        L = ctypes.CDLL(_LIB)
        i64 = ctypes.c_int64
        for name, args, res in (("rule_rows_tile", 3, ctypes.c_int), ("rule_weights_tile", 3, ctypes.c_int),
                                ("rule_tile_of", 2, ctypes.c_int), ("rule_few_rows", 2, ctypes.c_int),
                                ("rule_few_form", 3, ctypes.c_int), ("rule_row_tiles", 3, i64),
                                ("rule_tiles_over", 1, i64), ("rule_serve_rows", 3, ctypes.c_int),
                                ("rule_serve_parts", 3, ctypes.c_int), ("rule_shrink_parts", 3, ctypes.c_int),
                                ("rule_serve_many", 5, ctypes.c_int), ("rule_plan_serve_rows", 5, ctypes.c_int),
                                ("rule_few_rows_masked", 4, ctypes.c_int)):
            f = getattr(L, name)
            f.argtypes = [i64] * args
            f.restype = res
        L.rule_masked_small.argtypes = [ctypes.c_int, i64]
        _lib = L
    return _lib


def forward(rows, groups, cols):
    """("few", form) or ("tile", size) of a grouped product on whole rows."""
    L = rules()
    if L.rule_few_rows(rows, groups):
        return "few", L.rule_few_form(rows, groups, cols)
    return "tile", L.rule_rows_tile(rows, groups, cols)


def adapter(rows, n, k):
    """(tile size or None, rows in the few-row form) of an adapter product."""
    L = rules()
    serve = L.rule_serve_rows(rows, n, k)
    tiles = rows - serve
    up = lambda b: -(-tiles // b) * -(-n // b)  # noqa: E731
    return (L.rule_tile_of(up(128), up(256)) if tiles else None), serve


def adapter_of(rows, n, k, adapters, rank):
    """The same with the adapters and their rank, which move rows of many
    adapters into the few-row form."""
    L = rules()
    serve = L.rule_plan_serve_rows(rows, n, k, -(-rank // 16) * 16, adapters)
    tiles = rows - serve
    up = lambda b: -(-tiles // b) * -(-n // b)  # noqa: E731
    return (L.rule_tile_of(up(128), up(256)) if tiles else None), serve


def gram(count, side):
    """(tile size, tiles left to small ones) of a symmetric product."""
    L = rules()
    up = lambda b: count * -(-side // b) * (-(-side // b) + 1) // 2  # noqa: E731
    over = L.rule_tiles_over(up(256))
    return (LARGE if over else L.rule_tile_of(up(128), up(256))), over
