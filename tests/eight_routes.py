"""Which kernel an 8-bit product takes: the library's own rules
(paper_2609_09095_amd/csrc/eight_rules.hpp), compiled with g++ on first use, so that a
test of one form can assert that its sizes still reach it."""
from __future__ import annotations

import ctypes
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2609_09095_amd", "csrc")
_HOST = os.path.join(ROOT, "tests", "host")
_SRC = os.path.join(_HOST, "eight_plans.cpp")
_HDR = os.path.join(CSRC, "eight_rules.hpp")
_LIB = os.path.join(_HOST, "libeightplans.so")
_lib = None

FORMS = ["few16", "few32", "few48", "small", "middle", "large"]


def plans():
    global _lib
    if _lib is None:
        newest = max(os.path.getmtime(_SRC), os.path.getmtime(_HDR))
        if not os.path.exists(_LIB) or os.path.getmtime(_LIB) < newest:
            tmp = _LIB + ".tmp%d" % os.getpid()
            subprocess.check_call(["g++", "-O2", "-std=c++20", "-shared", "-fPIC", f"-I{CSRC}", "-o", tmp, _SRC])
            os.replace(tmp, _LIB)
        L = ctypes.CDLL(_LIB)
        i64, i32 = ctypes.c_int64, ctypes.c_int
        for name, args, res in (("plan_form", [i64, i64, i64, i32], i32), ("plan_split", [i64, i64, i64, i32], i32),
                                ("plan_tall", [i64, i64], i32), ("plan_room", [i64, i64, i64, i32], i64),
                                ("plan_words", [i64] * 4, i32), ("plan_dma", [i64] * 4, i32)):
            f = getattr(L, name)
            f.argtypes, f.restype = args, res
        _lib = L
    return _lib


def scaled_route(rows, n, k, squares, dtype, A, B):
    """The form's name, with its loads ("dma" or "masked") where it has tiles, and its
    parts, e.g. ("small", "masked", 4), for operands that lie as A and B do."""
    L = plans()
    at = (A.data_ptr(), A.stride(0), B.data_ptr(), B.stride(0))
    words, dma = L.plan_words(*at), L.plan_dma(*at)
    form, split = FORMS[L.plan_form(rows, n, k, words)], L.plan_split(rows, n, k, words)
    if form.startswith("few"):
        return form, "", split
    if not dma:
        return ("small" if form == "small" else "middle"), "masked", split
    if form != "small" and (dtype == "f32" or not squares):
        form = "tall" if split == 1 and L.plan_tall(rows, n) else "middle"
    return form, "dma", split
