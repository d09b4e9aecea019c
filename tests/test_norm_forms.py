"""The forms of the norm's kernels: each covers its row, the kernels have every one that
the rule gives and no other, and launches are no larger than the rule says."""
import os
import re

import pytest

from test_eight_rules import L  # noqa: F401  (the rules, compiled)

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
WIDTHS = sorted(set(range(1, 2100)) | set(range(2100, 32769, 61)) |
                {w + d for w in range(512, 32769, 512) for d in (-7, -1, 0, 1, 7) if w + d <= 32768})


def test_a_row_is_covered_and_no_chunk_idle(L):  # noqa: F811
    for width in WIDTHS:
        lanes, chunks = L.rule_norm_lanes(width), L.rule_norm_chunks(width)
        assert lanes * chunks * 8 >= width, width
        assert lanes * (chunks - 1) * 8 < width or (lanes, chunks) == (1024, 4), width


def test_kernels_of_every_form(L):  # noqa: F811
    with open(os.path.join(ROOT, "paper_2609_09095_amd", "csrc", "norm.hip")) as f:
        text = f.read()
    cases = re.findall(r"case (\d+) \* 8 \+ (\d+): return f\.template operator\(\)<(\d+), (\d+)>\(\);", text)
    assert all((a, b) == (c, d) for a, b, c, d in cases)
    assert {(int(a), int(b)) for a, b, _, _ in cases} == {(L.rule_norm_lanes(w), L.rule_norm_chunks(w)) for w in WIDTHS}
    assert re.search(r"default: return hipError\w+;", text)


@pytest.mark.parametrize("rows", [1, 2, 7, 300, 4000, 70001, 1 << 30])
def test_launches_fit_the_threads_of_a_cu(L, rows):  # noqa: F811
    """1536 threads a CU forward, 768 in the gradient, at least a block; 256 CUs."""
    for width in WIDTHS:
        threads = L.rule_norm_threads(width)
        need = -(-rows // (threads // L.rule_norm_lanes(width)))
        assert L.rule_norm_blocks(rows, width) == min(need, 256 * max(1, 1536 // threads))
        assert L.rule_norm_parts(rows, width) == min(need, 256 * max(1, 768 // threads))
