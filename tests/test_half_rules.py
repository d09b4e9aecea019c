"""The rules by which the 16-bit products choose their tiles, on the CPU: on
the faster side at sizes that were measured both ways, and within their
limits over all sizes."""
import itertools

from half_routes import FEW16, FEW32, FEW64X32, FEW64X64, LARGE, MIDDLE, SMALL, adapter, forward, gram, rules


def test_row_tiles_on_the_measured_side():
    L = rules()
    for c, want in (((16384, 16, 4096), LARGE), ((2048, 8, 4096), LARGE), ((20000, 2, 4096), LARGE),
                    ((4096, 1, 4096), LARGE), ((8192, 1, 8192), LARGE), ((2048, 8, 2048), MIDDLE),
                    ((4096, 8, 4096), MIDDLE), ((16384, 8, 1024), MIDDLE), ((1024, 8, 4096), MIDDLE),
                    ((4096, 32, 2048), MIDDLE), ((512, 8, 4096), SMALL), ((512, 8, 1024), SMALL), ((700, 2, 512), SMALL)):
        assert L.rule_rows_tile(*c) == want, c


def test_weight_tiles_on_the_measured_side():
    L = rules()
    for c, want in (((4096, 2048, 8), LARGE), ((4096, 2048, 16), LARGE), ((4096, 4096, 1), LARGE),
                    ((2048, 1024, 16), MIDDLE), ((4096, 2048, 2), MIDDLE), ((1024, 1024, 8), MIDDLE),
                    ((512, 256, 2), SMALL)):
        assert L.rule_weights_tile(*c) == want, c


def test_few_rows_on_the_measured_side():
    for c, want in (((2, 8, 2048), ("few", FEW16)), ((16, 1, 4096), ("few", FEW16)), ((40, 1, 4096), ("few", FEW32)),
                    ((256, 64, 1024), ("few", FEW64X32)), ((64, 8, 4096), ("few", FEW64X32)),
                    ((256, 8, 4096), ("few", FEW64X64)), ((512, 8, 4096), ("tile", SMALL))):
        assert forward(*c) == want, c


def test_few_rows_of_masked_operands_on_the_measured_side():
    L = rules()
    for c, want in (((960, 29, 1024, 1971), 0), ((3000, 64, 1000, 777), 0), ((500, 16, 3001, 3000), 0),
                    ((100, 29, 1024, 1971), 0), ((64, 8, 2048, 2047), 0), ((128, 8, 512, 513), 1),
                    ((300, 64, 4000, 777), 1), ((250, 16, 3001, 3000), 1), ((16, 1, 4096, 4095), 1),
                    ((1, 1, 1, 1), 1), ((16, 8, 2048, 2047), 1), ((17, 8, 2048, 2047), 0)):
        assert L.rule_few_rows_masked(*c) == want, c


def test_adapter_forms():
    assert adapter(1, 4096, 4096) == (None, 1) and adapter(128, 4096, 4096) == (None, 128)
    assert adapter(256, 1024, 1024) == (None, 256) and adapter(512, 1024, 1024) == (SMALL, 0)
    assert adapter(512, 4096, 4096) == (SMALL, 0)
    # 4 rows would cost the large tiles a round of their own, 100 rows are worth one
    assert adapter(4100, 4096, 4096) == (LARGE, 4) and adapter(4196, 4096, 4096)[1] == 0
    assert adapter(4100, 1024, 4096)[1] == 0  # a round has room for them


def test_many_adapters_in_few_rows():
    L = rules()
    for c, want in (((256, 4096, 4096, 16, 8), 1), ((256, 4096, 4096, 16, 7), 0), ((256, 4096, 4096, 64, 32), 1),
                    ((256, 4096, 4096, 64, 31), 0), ((256, 4096, 4096, 0, 8), 0), ((256, 4096, 4095, 16, 16), 0),
                    ((256, 4096, 4095, 16, 64), 1), ((512, 1024, 1024, 16, 16), 1),
                    ((512, 1024, 1024, 16, 15), 0), ((512, 2048, 2048, 64, 32), 1), ((512, 2048, 2048, 64, 31), 0),
                    ((512, 4096, 4096, 16, 65536), 0), ((512, 1 << 22, 1 << 22, 256, 65536), 0),
                    ((513, 1, 1, 16, 64), 0)):
        assert L.rule_serve_many(*c) == want, c


def test_adapter_plans_stay_within_their_limits():
    """Parts between 1 and 8 (the join holds 8), the few-row form's rows within
    a launch's grid, over all sizes."""
    L = rules()
    for rows, n, k in itertools.product((1, 15, 64, 128, 129, 257, 512, 513, 4100, 65536, 1 << 20, 1 << 30),
                                        (1, 7, 64, 1000, 4096, 1 << 22), (0, 1, 63, 512, 4096, 1 << 22)):
        serve = L.rule_serve_rows(rows, n, k)
        assert 0 <= serve <= 512 and serve <= rows
        assert (1 if serve else 0) <= L.rule_serve_parts(rows, n, k) <= 8
        assert 1 <= L.rule_shrink_parts(rows, n, k) <= 8


def test_symmetric_products_over_whole_rounds():
    assert gram(2, 4096) == (LARGE, 16) and gram(6, 2304) == (LARGE, 14)
    assert gram(1, 4096)[1] == 0 and gram(32, 128) == (SMALL, 0)
    L = rules()
    for large in range(1, 3000):
        over = L.rule_tiles_over(large)
        assert over == 0 or ((large - over) % 256 == 0 and large > over and over <= 48)


def test_expected_row_tiles():
    """At least the tiles that whole rows take and, while there are rows, one
    per group; never more than a launch is made for."""
    L = rules()
    for rows, groups, bm in itertools.product((1, 2, 63, 64, 65, 1000, 4096, 1 << 30), (1, 2, 8, 64, 65536), (64, 128, 256)):
        t = L.rule_row_tiles(rows, groups, bm)
        assert -(-rows // bm) <= t <= rows // bm + groups + 1 and t >= min(groups, rows)


def test_small_tiles_below_four_fifths_of_the_cus():
    L = rules()
    for c, want in (((1536, 1, 2048), SMALL), ((2048, 1, 2048), MIDDLE), ((3584, 2, 1024), MIDDLE),
                    ((512, 8, 4096), SMALL), ((640, 8, 4096), MIDDLE)):
        assert L.rule_rows_tile(*c) == want, c
    assert L.rule_weights_tile(2048, 1024, 2) == MIDDLE and L.rule_weights_tile(1024, 512, 6) == SMALL
