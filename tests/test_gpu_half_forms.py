"""Every form that the 16-bit products choose between, at sizes that reach it
by the library's own rules, against 64 bits (tolerances as in the tests of
each operator)."""
import numpy as np
import pytest
import torch

import gpu_util
import paper_2609_09095_amd as oz
from half_routes import (FEW16, FEW32, FEW64X32, FEW64X64, LARGE, MIDDLE, SMALL, adapter, forward, gram, rules)
from test_gpu_adapter import check as check_adapter
from test_gpu_grouped import check_all, close, draw
from test_gpu_orthogonalise import check as check_orth, gradient

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def gpu():
    gpu_util.require_gpu()


def sizes_of(rows, groups, seed=0):
    """Uneven groups, the second one empty where there are three or more."""
    rng = np.random.default_rng(seed)
    p = rng.random(groups) + 0.2
    if groups > 2:
        p[1] = 0
    return rng.multinomial(rows, p / p.sum()).tolist()


# rows, groups, n, k: the form of the forward product (n columns) and of the
# input's gradient (k columns; always whole tiles)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows, groups, n, k, fwd, dx", [
    (2, 8, 2048, 96, ("few", FEW16), SMALL), (17, 3, 200, 1000, ("few", FEW16), SMALL),
    (40, 1, 256, 333, ("few", FEW32), SMALL), (64, 8, 2056, 200, ("few", FEW64X32), SMALL),
    (300, 8, 2048, 72, ("few", FEW64X64), SMALL), (500, 2, 512, 136, ("tile", SMALL), SMALL),
    (4096, 4, 1024, 1032, ("tile", MIDDLE), MIDDLE), (2048, 2, 4096, 200, ("tile", LARGE), SMALL),
    (2048, 2, 200, 4096, ("tile", SMALL), LARGE),
])
def test_grouped_rows(dtype, rows, groups, n, k, fwd, dx):
    assert forward(rows, groups, n) == fwd and rules().rule_rows_tile(rows, groups, k) == dx
    check_all(rows, n, k, sizes_of(rows, groups), dtype)


@pytest.mark.parametrize("rows, groups, n, k, small", [(500, 2, 511, 77, True), (4096, 4, 1023, 1031, False)])
def test_grouped_rows_masked(rows, groups, n, k, small):
    for cols in (n, k):
        tiles = rules().rule_row_tiles(rows, groups, 128) * -(-cols // 128)
        assert bool(rules().rule_masked_small(0, tiles)) == small
    check_all(rows, n, k, sizes_of(rows, groups), torch.bfloat16)


# Few unaligned rows a group: straight into fragments or in tiles.
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows, groups, n, k, few", [
    (16, 8, 2057, 777, 1), (100, 8, 300, 129, 1), (300, 64, 700, 901, 1), (9, 1, 100, 1027, 1), (70, 8, 1000, 999, 0),
    (700, 29, 260, 1001, 0), (129, 8, 65, 7, 0)])
def test_few_rows_masked(dtype, rows, groups, n, k, few):
    assert rules().rule_few_rows(rows, groups) and rules().rule_few_rows_masked(rows, groups, n, k) == few
    check_all(rows, n, k, sizes_of(rows, groups), dtype)


# Unaligned operands of a long depth in few tiles: sets of wavefronts share it.
# Groups of fewer stages than sets (and of none) leave sets without a part.
@pytest.mark.parametrize("sizes, n, k", [([2100, 0, 1, 70, 130, 1700], 70, 65), ([641, 700], 129, 33), ([2000], 5, 3)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_weights_of_long_groups_masked(sizes, n, k, dtype):
    assert rules().rule_masked_sets(len(sizes) * -(-n // 64) * -(-k // 64), sum(sizes) // len(sizes))
    check_all(sum(sizes), n, k, sizes, dtype)


@pytest.mark.parametrize("rows, groups, n, k", [(300, 3, 129, 777), (200, 1, 641, 1500), (130, 2, 1001, 643)])
def test_rows_of_long_depths_masked(rows, groups, n, k):
    assert rules().rule_masked_sets(rules().rule_row_tiles(rows, groups, 64) * -(-n // 64), k)
    check_all(rows, n, k, sizes_of(rows, groups), torch.bfloat16)


def test_adapter_of_long_depths_masked():
    assert adapter(450, 600, 777)[1] == 0 and rules().rule_masked_sets(8 * 10, 777)
    check_adapter(450, 600, 777, 5, 20, ids_of(450, 5), torch.bfloat16)


@pytest.mark.parametrize("rows, groups, n, k, want", [(700, 2, 512, 256, SMALL), (900, 8, 1024, 1024, MIDDLE),
                                                       (900, 12, 2048, 2048, LARGE), (300, 1, 2048, 2304, MIDDLE),
                                                       (300, 1, 4096, 4096, LARGE)])
def test_grouped_weights(rows, groups, n, k, want):
    assert rules().rule_weights_tile(n, k, groups) == want
    check_all(rows, n, k, sizes_of(rows, groups), torch.bfloat16)


@pytest.mark.parametrize("n, k, groups, small", [(511, 129, 3, True), (1023, 1025, 8, False)])
def test_grouped_weights_masked(n, k, groups, small):
    assert bool(rules().rule_masked_small(1, groups * -(-n // 128) * -(-k // 128))) == small
    check_all(600, n, k, sizes_of(600, groups), torch.bfloat16)


@pytest.mark.parametrize("groups", [63, 64, 65, 255, 256, 300, 1000])
@pytest.mark.parametrize("rows", [90, 20000])
def test_many_groups(groups, rows):
    """Up to 255 groups are held in registers, more are read again."""
    check_all(rows, 72, 64, sizes_of(rows, groups), torch.bfloat16)


@pytest.mark.parametrize("k", [64, 61])
def test_offsets_past_32_bits(k):
    """Rows of an activation and matrices of a stack more than 2^32 elements
    from the first one."""
    rows, n, pitch = 700, 48, 1 << 23
    f = dict(dtype=torch.bfloat16, device="cuda")
    wide = torch.empty(rows, pitch, **f)
    assert wide.numel() > 1 << 32
    X = wide[:, 5:5 + k]
    X.copy_(draw((rows, k), torch.bfloat16, 1))
    stack = torch.empty(3, 1 << 32, **f)
    W = stack[:, :n * k].view(3, n, k)
    W.copy_(draw((3, n, k), torch.bfloat16, 2))
    E = torch.tensor([200, 300, 700], dtype=torch.int32, device="cuda")
    out = torch.empty(rows, pitch, **f)
    Y = oz.ozaki25_grouped_matmul(X, W, E, out[:, 3:3 + n])
    dX = oz.ozaki25_grouped_matmul_dx(Y, W, E)
    dW = oz.ozaki25_grouped_matmul_dw(Y, X, E, torch.empty(3, 1 << 31, device="cuda")[:, :n * k].view(3, n, k))
    torch.cuda.synchronize()
    for g, (i, j) in enumerate([(0, 200), (200, 300), (300, 700)]):
        x, w, y = X[i:j].double(), W[g].double(), Y[i:j].double()
        close(Y[i:j], x @ w.t(), x.abs() @ w.abs().t(), k)
        close(dX[i:j], y @ w, y.abs() @ w.abs(), n)
        close(dW[g], y.t() @ x, y.abs().t() @ x.abs(), j - i)


def ids_of(rows, adapters):
    return np.sort(np.random.default_rng(rows).integers(-1, adapters, rows))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows, n, k, tile, serve", [
    (1, 300, 4096, None, 1), (20, 300, 600, None, 20), (64, 300, 600, None, 64), (100, 300, 600, None, 100),
    (300, 200, 600, None, 300), (400, 1024, 256, SMALL, 0), (2304, 2048, 136, MIDDLE, 0), (4096, 4096, 128, LARGE, 0),
    (4100, 4096, 128, LARGE, 4),
])
def test_adapter_forms(dtype, rows, n, k, tile, serve):
    assert adapter(rows, n, k) == (tile, serve)
    check_adapter(rows, n, k, 5, 24, ids_of(rows, 5), dtype)


# Rows of many adapters, each its own choice: few of them in the few-row form,
# more in tiles that go through up to 64 adapters each.
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows, n, k, adapters, rank, many", [
    (129, 4100, 520, 16, 24, 1), (256, 2056, 777, 70, 130, 1), (250, 2056, 777, 12, 24, 0), (255, 2056, 777, 130, 256, 1), (333, 1000, 1111, 16, 16, 1),
    (512, 1024, 264, 64, 65, 1), (500, 1025, 264, 15, 8, 0), (512, 3000, 4096, 64, 16, 0)])
def test_many_adapters(dtype, rows, n, k, adapters, rank, many):
    assert rules().rule_serve_many(rows, n, k, -(-rank // 16) * 16, adapters) == many
    ids = np.random.default_rng(rows).integers(-1, adapters + 1, rows)
    check_adapter(rows, n, k, adapters, rank, ids, dtype)


# The products X A^T in tiles: ranks that fill no tile of 64, rows of many
# adapters in any order, depths that end inside a stage.
@pytest.mark.parametrize("rows, n, k, rank, order", [
    (1024, 264, 520, 1, "any"), (1031, 520, 2056, 65, "any"), (1100, 512, 1032, 24, "sorted"),
    (2049, 136, 8, 128, "any"), (1087, 264, 1096, 200, "sorted")])
def test_adapter_many_rows(rows, n, k, rank, order):
    ids = ids_of(rows, 9)
    if order == "any":
        ids = np.random.default_rng(rank).permutation(ids)
    check_adapter(rows, n, k, 9, rank, ids, torch.bfloat16)


@pytest.mark.parametrize("rows, n, k, small", [(400, 1000, 111, True), (2048, 2049, 137, False)])
def test_adapter_masked(rows, n, k, small):
    assert bool(rules().rule_masked_small(0, -(-rows // 128) * -(-n // 128))) == small
    check_adapter(rows, n, k, 5, 20, ids_of(rows, 5), torch.bfloat16)


@pytest.mark.parametrize("count, m, n, tile, over", [
    (2, 136, 200, SMALL, 0), (4, 1536, 1600, MIDDLE, 0), (2, 3000, 4100, LARGE, 0), (6, 2304, 2310, LARGE, 14),
    (6, 2310, 2304, LARGE, 14),
])
def test_orthogonalise_tiles(count, m, n, tile, over):
    assert gram(count, -(-min(m, n) // 8) * 8) == (tile, over)
    check_orth(gradient((count, m, n), torch.float32))
