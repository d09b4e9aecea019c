"""What the 16-bit products refuse, before anything is launched: the C entry
points with addresses that are never read, and the binding with CPU tensors
(shapes and sizes are checked before the device)."""
import ctypes

import pytest
import torch

import paper_2609_09095_amd as oz

OK, BAD, UNSUPPORTED, ROOM = oz.SUCCESS, oz.ERR_INVALID_VALUE, oz.ERR_UNSUPPORTED, oz.ERR_WORKSPACE
BF = oz.BF16


@pytest.fixture(scope="module", autouse=True)
def built_library():
    import os
    if not os.path.exists(oz.library_path()):
        from paper_2609_09095_amd import build
        build.build()
    oz.lib()


def p(i):
    """The i-th of addresses far apart."""
    return ctypes.c_void_p(i << 32)


def rows_call(f, rows=8, n=16, k=32, groups=2, X=p(1), ldx=None, W=p(2), ldw=None, stride=None, ends=p(3), Y=p(4),
              ldy=None, type=BF, dx=False):
    into, out = (n, k) if dx else (k, n)
    return f(rows, n, k, groups, X, into if ldx is None else ldx, W, k if ldw is None else ldw,
             n * k if stride is None else stride, ends, Y, out if ldy is None else ldy, type, None)


@pytest.mark.parametrize("dx", [False, True])
def test_grouped_rows_refusals(dx):
    f = oz.lib().ozaki25_grouped_matmul_dx if dx else oz.lib().ozaki25_grouped_matmul
    into, out = (16, 32) if dx else (32, 16)

    def call(**kw):
        return rows_call(f, dx=dx, **kw)

    for kw in (dict(rows=-1), dict(n=-1), dict(k=-1), dict(groups=-1), dict(ldx=into - 1), dict(ldw=31), dict(ldy=out - 1),
               dict(ldx=oz.MAX_LD + 1), dict(stride=-1), dict(X=None), dict(W=None), dict(ends=None), dict(Y=None),
               dict(X=ctypes.c_void_p((1 << 32) + 1)), dict(Y=ctypes.c_void_p((4 << 32) + 1)),
               dict(ends=ctypes.c_void_p((3 << 32) + 2)), dict(type=oz.F32), dict(type=7),
               dict(Y=p(1)), dict(Y=ctypes.c_void_p((1 << 32) + 16)), dict(Y=p(2)), dict(Y=p(3))):
        assert call(**kw) == BAD, kw
    assert call(rows=oz.MAX_ROWS + 1) == UNSUPPORTED and call(groups=oz.MAX_GROUPS + 1) == UNSUPPORTED
    wide = oz.MAX_WIDTH + 1
    assert rows_call(f, n=wide, dx=dx) == UNSUPPORTED and rows_call(f, k=wide, dx=dx) == UNSUPPORTED
    # more output tiles than a launch holds
    assert rows_call(f, rows=oz.MAX_ROWS, n=1 << 16, k=1 << 16, X=p(1 << 18), W=p(1 << 20), Y=p(1 << 22), dx=dx) == UNSUPPORTED
    # nothing to do
    assert call(rows=0, X=None, Y=None) == OK
    assert rows_call(f, n=16 if dx else 0, k=0 if dx else 32, X=None, W=None, Y=None, dx=dx, ldw=32, ldy=1) == OK


def test_grouped_weights_refusals():
    f = oz.lib().ozaki25_grouped_matmul_dw

    def call(rows=8, n=16, k=32, groups=2, dY=p(1), lddy=16, X=p(2), ldx=32, ends=p(3), dW=p(4), lddw=32, stride=512,
             type=BF, out=BF):
        return f(rows, n, k, groups, dY, lddy, X, ldx, ends, dW, lddw, stride, type, out, None)

    for kw in (dict(rows=-1), dict(n=-1), dict(k=-1), dict(groups=-1), dict(lddy=15), dict(ldx=31), dict(lddw=31),
               dict(stride=511), dict(dY=None), dict(X=None), dict(ends=None), dict(dW=None), dict(type=oz.F32),
               dict(out=oz.F16), dict(out=9), dict(out=oz.F32, dW=ctypes.c_void_p((4 << 32) + 2)), dict(dW=p(1)),
               dict(dW=p(2)), dict(dW=p(3))):
        assert call(**kw) == BAD, kw
    assert call(rows=oz.MAX_ROWS + 1) == UNSUPPORTED and call(groups=oz.MAX_GROUPS + 1) == UNSUPPORTED
    assert call(groups=0, dW=None) == OK and call(n=0, dW=None, lddy=1) == OK and call(k=0, dW=None) == OK


def test_adapter_refusals():
    f = oz.lib().ozaki25_adapter_matmul
    need = oz.ozaki25_adapter_matmul_workspace_size(8, 16, 32, 3, 4)
    assert need > 0 and need % 256 == 0

    def call(rows=8, n=16, k=32, adapters=3, rank=4, X=p(1), ldx=32, W=p(2), ldw=32, ids=p(3), A=p(4), lda=32, sa=128,
             B=p(5), ldb=4, sb=64, scales=None, Y=p(6), ldy=16, type=BF, room=p(7), size=need):
        return f(rows, n, k, adapters, rank, X, ldx, W, ldw, ids, A, lda, sa, B, ldb, sb, scales, Y, ldy, type, room, size,
                 None)

    for kw in (dict(rows=-1), dict(n=-1), dict(k=-1), dict(adapters=-1), dict(rank=-1), dict(ldx=31), dict(ldw=31),
               dict(lda=31), dict(ldb=3), dict(ldy=15), dict(sa=-1), dict(sb=-1), dict(X=None), dict(W=None),
               dict(ids=None), dict(A=None), dict(B=None), dict(Y=None), dict(type=oz.F32), dict(Y=p(1)), dict(Y=p(2)),
               dict(Y=p(3)), dict(Y=p(4)), dict(Y=p(5)), dict(room=p(6)), dict(room=p(1)),
               dict(scales=ctypes.c_void_p((9 << 32) + 2)), dict(scales=p(6)),
               dict(room=ctypes.c_void_p((7 << 32) + 128))):
        assert call(**kw) == BAD, kw
    assert call(rank=oz.MAX_RANK + 1, ldb=oz.MAX_RANK + 1) == UNSUPPORTED
    assert call(rows=oz.MAX_ROWS + 1) == UNSUPPORTED
    assert call(size=need - 1) == ROOM
    assert call(rows=0, X=None, Y=None) == OK and call(n=0, W=None, Y=None) == OK
    # more work-items than a launch holds, before anything runs
    big = oz.ozaki25_adapter_matmul_workspace_size(oz.MAX_ROWS, 1, 1, 1, 1)
    assert call(rows=oz.MAX_ROWS, n=1, k=1, adapters=1, rank=1, W=p(1 << 8), ids=p(1 << 9), A=p(1 << 10), B=p(1 << 11),
                Y=p(1 << 12), room=p(1 << 13), size=big) == UNSUPPORTED
    assert oz.ozaki25_adapter_matmul_workspace_size(8, 16, 32, 3, oz.MAX_RANK + 1) == 0
    assert oz.ozaki25_adapter_matmul_workspace_size(-1, 16, 32, 3, 4) == 0


def test_orthogonalise_refusals():
    f = oz.lib().ozaki25_orthogonalise
    need = oz.ozaki25_orthogonalise_workspace_size(2, 200, 136)
    assert need >= 2 * 200 * 136 * 8 and need % 256 == 0

    def call(count=2, m=200, n=136, G=p(1), ldg=136, sg=27200, type=oz.F32, X=p(2), ldx=136, sx=27200, steps=5, a=3.0, b=-4.0,
             c=2.0, eps=1e-7, room=p(3), size=need):
        return f(count, m, n, G, ldg, sg, type, X, ldx, sx, steps, a, b, c, eps, room, size, None)

    inf, nan = float("inf"), float("nan")
    for kw in (dict(count=-1), dict(m=-1), dict(n=-1), dict(ldg=135), dict(ldx=135), dict(sg=-1), dict(sx=27199),
               dict(type=5), dict(steps=0), dict(steps=oz.MAX_STEPS + 1), dict(a=nan), dict(b=inf), dict(c=-inf), dict(eps=-1.0),
               dict(eps=nan), dict(eps=inf), dict(G=None), dict(X=None), dict(G=ctypes.c_void_p((1 << 32) + 2)), dict(X=p(1)),
               dict(room=p(1)), dict(room=p(2)), dict(room=ctypes.c_void_p((3 << 32) + 64))):
        assert call(**kw) == BAD, kw
    side = oz.MAX_SIDE + 1
    assert call(m=side, sx=side * 136) == UNSUPPORTED and call(n=side, ldg=side, ldx=side, sx=200 * side) == UNSUPPORTED
    assert call(count=oz.MAX_GROUPS) == UNSUPPORTED
    assert call(size=need - 1) == ROOM
    assert call(count=0, G=None) == OK and call(m=0, G=None) == OK and call(n=0, X=None) == OK
    assert oz.ozaki25_orthogonalise_workspace_size(2, side, 4) == 0 == oz.ozaki25_orthogonalise_workspace_size(0, 4, 4)


def bf(*shape):
    return torch.zeros(shape, dtype=torch.bfloat16)


def i32(*shape):
    return torch.zeros(shape, dtype=torch.int32)


def raises(match, fn, *a, **kw):
    with pytest.raises(ValueError, match=match):
        fn(*a, **kw)


def test_binding_grouped():
    f, x, w = oz.ozaki25_grouped_matmul, oz.ozaki25_grouped_matmul_dx, oz.ozaki25_grouped_matmul_dw
    raises("X must be a 2-D tensor", f, bf(4, 8).float(), bf(2, 6, 8), i32(2))
    raises("X must be a 2-D tensor", f, bf(4, 8, 1), bf(2, 6, 8), i32(2))
    raises("W must be a 3-D tensor", f, bf(4, 8), bf(2, 6, 8).half(), i32(2))
    raises("W has 7 columns", f, bf(4, 8), bf(2, 6, 7), i32(2))
    raises("ends holds 3", f, bf(4, 8), bf(2, 6, 8), i32(3))
    raises("ends must be", f, bf(4, 8), bf(2, 6, 8), torch.zeros(2))
    raises("ends must be", f, bf(4, 8), bf(2, 6, 8), [1, 2])
    raises(r"Y has shape \(4, 5\)", f, bf(4, 8), bf(2, 6, 8), i32(2), bf(4, 5))
    raises("row-major", f, bf(8, 4).t(), bf(2, 6, 8), i32(2))
    raises("rows overlap", f, bf(8).expand(4, 8), bf(2, 6, 8), i32(2))
    raises("CUDA tensor", f, bf(4, 8), bf(2, 6, 8), i32(2))
    raises("W has 5 rows", x, bf(4, 6), bf(2, 5, 8), i32(2))
    raises(r"dX has shape", x, bf(4, 6), bf(2, 6, 8), i32(2), bf(4, 6))
    raises("CUDA tensor", x, bf(4, 6), bf(2, 6, 8), i32(2))
    raises("X has 5 rows", w, bf(4, 6), bf(5, 8), i32(2))
    raises("dW has dtype", w, bf(4, 6), bf(4, 8), i32(2), bf(2, 6, 8), torch.float32)
    raises("dW must be", w, bf(4, 6), bf(4, 8), i32(2), out_dtype=torch.float16)
    raises("ends must be", w, bf(4, 6), bf(4, 8), None)
    raises("CUDA tensor", w, bf(4, 6), bf(4, 8), i32(2))


def test_binding_adapter():
    f = oz.ozaki25_adapter_matmul
    X, W, ids, A, B = bf(4, 8), bf(6, 8), i32(4), bf(3, 2, 8), bf(3, 6, 2)
    raises("W has 7 columns", f, X, bf(6, 7), ids, A, B)
    raises("A has 7 columns", f, X, W, ids, bf(3, 2, 7), B)
    raises(r"B has shape \(3, 6, 3\)", f, X, W, ids, A, bf(3, 6, 3))
    raises("ids holds 5", f, X, W, i32(5), A, B)
    raises("ids must be", f, X, W, ids.long(), A, B)
    raises("scales must be", f, X, W, ids, A, B, torch.zeros(3, dtype=torch.float64))
    raises("scales holds 4", f, X, W, ids, A, B, torch.zeros(4))
    raises("workspace must be", f, X, W, ids, A, B, workspace=torch.zeros(9))
    raises("Y must be", f, X, W, ids, A, B, Y=bf(4, 6).half())
    raises("CUDA tensor", f, X, W, ids, A, B)


def test_binding_orthogonalise():
    f = oz.ozaki25_orthogonalise
    raises("2-D or 3-D", f, bf(8))
    raises("G must be", f, torch.zeros(4, 4, dtype=torch.float64))
    raises("row-major", f, bf(4, 8).t())
    raises(r"X has shape \(4, 7\)", f, bf(4, 8), bf(4, 7))
    raises("X must be", f, bf(4, 8), torch.zeros(4, 8))
    raises("workspace must be", f, bf(4, 8), workspace=torch.zeros(9))
    with pytest.raises(ValueError):
        f(bf(4, 8), coefficients=(1.0, 2.0))
