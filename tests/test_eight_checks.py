"""What the operators of the 8-bit path refuse, before anything is launched: the C
entry points with addresses that are never read, and the binding with CPU
tensors."""
import ctypes
import struct

import pytest
import torch

import paper_2609_09095_amd as oz

OK, BAD, UNSUPPORTED, ROOM = oz.SUCCESS, oz.ERR_INVALID_VALUE, oz.ERR_UNSUPPORTED, oz.ERR_WORKSPACE
BF = oz.BF16
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module", autouse=True)
def built_library():
    import os
    if not os.path.exists(oz.library_path()):
        from paper_2609_09095_amd import build
        build.build()
    oz.lib()


def p(i, off=0):
    """The i-th of addresses far apart."""
    return ctypes.c_void_p((i << 32) + off)


def raises(match, fn, *a, **kw):
    with pytest.raises(ValueError, match=match):
        fn(*a, **kw)


def test_norm_refusals():
    f = oz.lib().ozaki25_rms_norm

    def call(rows=8, width=300, X=p(1), ldx=300, R=p(2), ldr=300, w=p(3), type=BF, eps=1e-6, H=p(4), ldh=300, Y=p(5),
             ldy=300, s=p(6), lds=8):
        return f(rows, width, X, ldx, R, ldr, w, type, eps, H, ldh, Y, ldy, s, lds, None)

    for kw in (dict(rows=-1), dict(width=-1), dict(ldx=299), dict(ldr=299), dict(ldh=299), dict(ldy=299), dict(lds=7),
               dict(type=3), dict(type=-1), dict(eps=-1.0), dict(eps=NAN), dict(eps=INF), dict(X=None), dict(Y=None),
               dict(H=None), dict(R=None), dict(X=p(1, 1)), dict(R=p(2, 1)), dict(w=p(3, 1)), dict(H=p(4, 1)), dict(s=p(6, 2)),
               dict(Y=p(5, 1), s=None), dict(type=oz.F32, X=p(1, 2)), dict(ldx=oz.MAX_LD + 1),
               # overlaps: the sum may only take the whole place of a part, the others none
               dict(H=p(1), ldh=301), dict(H=p(1, 2)), dict(H=p(2, 600)), dict(H=p(3)), dict(Y=p(1)), dict(Y=p(2)), dict(Y=p(3)),
               dict(Y=p(4)), dict(Y=p(6)), dict(s=p(1)), dict(s=p(4)), dict(X=p(1), R=p(1), H=p(1, 2))):
        assert call(**kw) == BAD, kw
    wide = oz.MAX_NORM_WIDTH + 1
    assert call(width=wide, ldx=wide, ldr=wide, ldh=wide, ldy=wide) == UNSUPPORTED
    assert call(rows=oz.MAX_ROWS + 1, lds=oz.MAX_ROWS + 1) == UNSUPPORTED
    assert call(rows=0, X=None, Y=None, H=None) == OK and call(width=0, X=None, Y=None) == OK


def test_norm_backward_refusals():
    f = oz.lib().ozaki25_rms_norm_backward
    need = oz.ozaki25_rms_norm_backward_workspace_size(8, 300)
    assert need > 0 and need % 256 == 0
    assert oz.ozaki25_rms_norm_backward_workspace_size(0, 300) == 0 == oz.ozaki25_rms_norm_backward_workspace_size(8, -1)

    def call(rows=8, width=300, Y=p(1), ldy=300, H=p(2), ldh=300, w=p(3), D=p(4), ldd=300, type=BF, eps=1e-6, X=p(5), ldx=300,
             g=p(6), room=p(7), size=need):
        return f(rows, width, Y, ldy, H, ldh, w, D, ldd, type, eps, X, ldx, g, room, size, None)

    for kw in (dict(rows=-1), dict(width=-1), dict(ldy=299), dict(ldh=299), dict(ldd=299), dict(ldx=299), dict(type=5),
               dict(eps=-1.0), dict(eps=NAN), dict(Y=None), dict(H=None), dict(X=None), dict(g=None), dict(Y=p(1, 1)),
               dict(H=p(2, 1)), dict(w=p(3, 1)), dict(D=p(4, 1)), dict(X=p(5, 1)), dict(g=p(6, 2)), dict(X=p(1), ldx=301),
               dict(X=p(1, 2)), dict(X=p(4, 2)), dict(X=p(2)), dict(X=p(3)), dict(g=p(1)), dict(g=p(2)), dict(g=p(5)),
               dict(room=p(7, 128)), dict(room=p(1)), dict(room=p(5)), dict(room=p(6))):
        assert call(**kw) == BAD, kw
    assert call(size=need - 1) == ROOM
    wide = oz.MAX_NORM_WIDTH + 1
    assert call(width=wide, ldy=wide, ldh=wide, ldd=wide, ldx=wide) == UNSUPPORTED
    assert call(width=0, g=None) == OK


def test_quantise_refusals():
    f = oz.lib().ozaki25_quantise

    def call(count=2, rows=8, cols=300, X=p(1), ldx=300, xs=2400, type=BF, squares=0, Q=p(2), ldq=304, qs=2432, s=p(3),
             T=p(4), ldt=16, ts=4800, st=p(5)):
        return f(count, rows, cols, X, ldx, xs, type, squares, Q, ldq, qs, s, T, ldt, ts, st, None)

    for kw in (dict(count=-1), dict(rows=-1), dict(cols=-1), dict(ldx=299), dict(ldq=299), dict(ldt=7), dict(type=3),
               dict(squares=2), dict(xs=-1), dict(qs=2427), dict(ts=4791), dict(X=None), dict(Q=None), dict(s=None), dict(T=None),
               dict(st=None), dict(Q=None, s=None, T=None, st=None), dict(X=p(1, 1)), dict(s=p(3, 2)), dict(st=p(5, 1)),
               dict(Q=p(1)), dict(T=p(1)), dict(s=p(1)), dict(st=p(1)), dict(Q=p(4)), dict(s=p(5)), dict(Q=p(3)), dict(T=p(5))):
        assert call(**kw) == BAD, kw
    assert call(count=oz.MAX_GROUPS) == UNSUPPORTED and call(rows=oz.MAX_ROWS + 1, ldt=oz.MAX_ROWS + 1) == UNSUPPORTED
    wide = oz.MAX_WIDTH + 1
    assert call(cols=wide, ldx=wide, ldq=wide) == UNSUPPORTED
    # more tiles than a launch holds
    assert call(count=1, rows=1 << 30, cols=1 << 12, ldx=1 << 12, X=p(1 << 12), Q=p(1 << 14), ldq=1 << 12, s=p(1 << 15), T=None,
                st=None) == UNSUPPORTED
    assert call(rows=0, X=None) == OK and call(count=0) == OK and call(cols=0, ldq=1) == OK


def test_scaled_matmul_refusals():
    f = oz.lib().ozaki25_scaled_matmul

    def call(rows=300, n=200, k=1000, A=p(1), lda=1000, a=p(2), ldas=300, B=p(3), ldb=1000, b=p(4), ldbs=None, squares=1, Y=p(5),
             ldy=200, out=BF, room=p(6), size=1 << 40):
        ldbs = (8 if squares else 200) if ldbs is None else ldbs
        return f(rows, n, k, A, lda, a, ldas, B, ldb, b, ldbs, squares, Y, ldy, out, room, size, None)

    for kw in (dict(rows=-1), dict(n=-1), dict(k=-1), dict(lda=999), dict(ldb=999), dict(ldas=299), dict(ldbs=7),
               dict(squares=0, ldbs=199), dict(squares=2), dict(ldy=199), dict(out=3), dict(out=-1), dict(A=None), dict(a=None),
               dict(B=None), dict(b=None), dict(Y=None), dict(a=p(2, 2)), dict(b=p(4, 1)), dict(Y=p(5, 1)),
               dict(Y=p(5, 2), out=oz.F32), dict(Y=p(1)), dict(Y=p(2)), dict(Y=p(3)), dict(Y=p(4)), dict(lda=oz.MAX_LD + 1)):
        assert call(**kw) == BAD, kw
    wide = oz.MAX_WIDTH + 1
    assert call(n=wide, ldy=wide, squares=0, ldbs=wide) == UNSUPPORTED and call(k=wide, lda=wide, ldb=wide, ldbs=wide) == UNSUPPORTED
    assert call(rows=oz.MAX_ROWS + 1, ldas=oz.MAX_ROWS + 1) == UNSUPPORTED
    assert call(rows=1 << 30, n=1 << 22, k=1, lda=1, ldb=1, ldas=1 << 30, ldbs=1, ldy=1 << 22, a=p(64), B=p(128), b=p(129),
                Y=p(1 << 25)) == UNSUPPORTED
    assert call(rows=0, A=None, Y=None) == OK and call(n=0, B=None, Y=None) == OK


def test_binding_scaled_matmul():
    A, B = torch.zeros(4, 300).to(torch.float8_e4m3fn), torch.zeros(200, 300).to(torch.float8_e4m3fn)
    a, b = torch.ones(3, 4), torch.ones(2, 3)
    f = oz.ozaki25_scaled_matmul
    raises("A must be", f, A.float(), a, B, b)
    raises("B has 299 columns", f, A, a, B[:, :299], b)
    raises("a_scales has shape", f, A, a[:2], B, b)
    raises("b_scales has shape", f, A, a, B, torch.ones(3, 200))
    raises("b_scales has shape", f, A, a, B, b, squares=False)
    raises("b_scales must be", f, A, a, B, b.double())
    raises("Y has dtype", f, A, a, B, b, out_dtype=torch.float16, Y=torch.zeros(4, 200))
    raises("out_dtype must be", f, A, a, B, b, out_dtype=torch.float64)
    raises("Y has shape", f, A, a, B, b, Y=torch.zeros(4, 201))
    raises("must be a CUDA tensor", f, A, a, B, b)


def test_expert_layer_refusals():
    f = oz.lib().ozaki25_expert_layer
    size = oz.ozaki25_expert_layer_workspace_size
    need = size(20, 2, 300, 200, 400)
    assert need > 0 and need % 256 == 0
    assert size(0, 2, 300, 200, 400) == 0 == size(20, 0, 300, 200, 400) == size(257, 2, 300, 200, 400) == size(20, 33, 300, 200, 400)

    def stack(w, ld, stride, s=0, lds=1, ss=0):
        return struct.pack("6q", w or 0, ld, stride, s, lds, ss)

    def call(tokens=20, top=2, experts=8, width=300, inner=200, out=400, X=p(1), ldx=300, which=p(2), gates=p(3), up=None, gate=None,
             down=None, Y=p(7), ldy=400, type=BF, room=p(8), size=need, no=()):
        up = up or stack(4 << 32, 300, 60000)
        gate = gate or stack(5 << 32, 300, 60000)
        down = down or stack(6 << 32, 200, 80000)
        at = [None if n in no else v for n, v in (("up", up), ("gate", gate), ("down", down))]
        return f(tokens, top, experts, width, inner, out, X, ldx, which, gates, *at, Y, ldy, type, room, size, None)

    eight = dict(up=stack(4 << 32, 300, 60000, 9 << 32, 3, 6), gate=stack(5 << 32, 300, 60000, 10 << 32, 3, 6),
                 down=stack(6 << 32, 200, 80000, 11 << 32, 2, 8))
    for kw in (dict(tokens=-1), dict(top=-1), dict(experts=-1), dict(width=-1), dict(inner=-1), dict(out=-1), dict(ldx=299),
               dict(ldy=399), dict(type=oz.F32), dict(type=4), dict(X=None), dict(which=None), dict(gates=None), dict(Y=None),
               dict(X=p(1, 1)), dict(which=p(2, 2)), dict(gates=p(3, 1)), dict(Y=p(7, 1)), dict(no=("up",)), dict(no=("down",)),
               dict(up=stack(None, 300, 60000)), dict(up=stack((4 << 32) + 1, 300, 60000)), dict(up=stack(4 << 32, 299, 60000)),
               dict(down=stack(6 << 32, 199, 80000)), dict(gate=stack(5 << 32, 300, -1)), dict(eight, gate=stack(5 << 32, 300, 60000)),
               dict(eight, down=stack(6 << 32, 200, 80000)), dict(eight, up=stack(4 << 32, 300, 60000, 9 << 32, 2, 6)),
               dict(eight, up=stack(4 << 32, 300, 60000, (9 << 32) + 2, 3, 6)), dict(eight, up=stack(4 << 32, 300, 60000, 9 << 32, 3, -1)),
               dict(Y=p(1)), dict(Y=p(2)), dict(Y=p(3)), dict(Y=p(4)), dict(Y=p(5)), dict(Y=p(6)), dict(Y=p(8)), dict(eight, Y=p(9)),
               dict(room=p(8, 64)), dict(room=p(1)), dict(room=p(4)), dict(eight, room=p(11))):
        assert call(**kw) == BAD, kw
    assert call(size=need - 1) == ROOM
    assert call(tokens=257) == UNSUPPORTED and call(top=33) == UNSUPPORTED and call(experts=4097) == UNSUPPORTED
    wide = oz.MAX_WIDTH + 1
    assert call(width=wide, ldx=wide, up=stack(4 << 32, wide, 0), gate=stack(5 << 32, wide, 0)) == UNSUPPORTED
    assert call(out=wide, ldy=wide) == UNSUPPORTED and call(inner=wide, down=stack(6 << 32, wide, 0)) == UNSUPPORTED
    assert call(tokens=0, X=None, Y=None) == OK and call(out=0, Y=None) == OK


def test_binding_expert_layer():
    H = torch.bfloat16
    X, up, down = torch.zeros(4, 20, dtype=H), torch.zeros(3, 16, 20, dtype=H), torch.zeros(3, 24, 16, dtype=H)
    which, gates = torch.zeros(4, 2, dtype=torch.int32), torch.zeros(4, 2)
    f = oz.ozaki25_expert_layer
    raises("X must be", f, X.float(), which, gates, up, down)
    raises("which must be", f, X, which.long(), gates, up, down)
    raises("which must be", f, X, which[:, 0], gates, up, down)
    raises("which has shape", f, X, which[:3], gates, up, down)
    raises("gates has shape", f, X, which, gates[:, :1].contiguous(), up, down)
    raises("gates must be", f, X, which, gates.to(H), up, down)
    raises("up must be", f, X, which, gates, up.float(), down)
    raises("up has 19 columns", f, X, which, gates, up[:, :, :19], down)
    raises("down has shape", f, X, which, gates, up, down[:2])
    raises("down has shape", f, X, which, gates, up, down[:, :, :15])
    raises("gate has shape", f, X, which, gates, up, down, gate=up[:, :15])
    raises("either all", f, X, which, gates, up, down, up_scales=torch.ones(3, 1, 1))
    raises("gate_scales need", f, X, which, gates, up, down, gate_scales=torch.ones(3, 1, 1))
    e = dict(up_scales=torch.ones(3, 1, 1), down_scales=torch.ones(3, 1, 1))
    raises("up must be", f, X, which, gates, up, down, **e)
    q, d = up.to(torch.float8_e4m3fn), down.to(torch.float8_e4m3fn)
    raises("up_scales has shape", f, X, which, gates, q, d, **dict(e, up_scales=torch.ones(3, 1, 2)))
    raises("Y has shape", f, X, which, gates, up, down, Y=X)
    raises("workspace must be", f, X, which, gates, up, down, workspace=X)
    raises("must be a CUDA tensor", f, X, which, gates, up, down)
    raises("must be a CUDA tensor", f, X, which, gates, q, d, **e)


def test_binding_norm():
    X, w = torch.zeros(4, 20, dtype=torch.bfloat16), torch.ones(20, dtype=torch.bfloat16)
    raises("X must be a 2-D", oz.ozaki25_rms_norm, X[0], w)
    raises("X must be a 2-D", oz.ozaki25_rms_norm, X.double(), w)
    raises("unit column stride", oz.ozaki25_rms_norm, X.t(), w)
    raises("weight must be", oz.ozaki25_rms_norm, X, w.float())
    raises("weight holds 19", oz.ozaki25_rms_norm, X, w[:19])
    raises("residual has shape", oz.ozaki25_rms_norm, X, w, residual=X[:3])
    raises("residual must be", oz.ozaki25_rms_norm, X, w, residual=X.float())
    raises("H needs a residual", oz.ozaki25_rms_norm, X, w, H=X)
    raises("scales need", oz.ozaki25_rms_norm, X, w, scales=torch.zeros(1, 4))
    raises("Y must be", oz.ozaki25_rms_norm, X, w, Y=X.float())
    raises("Y must be", oz.ozaki25_rms_norm, X, w, quantised=True, Y=X)
    raises("scales has shape", oz.ozaki25_rms_norm, X, w, quantised=True, scales=torch.zeros(4, 1))
    raises("must be a CUDA tensor", oz.ozaki25_rms_norm, X, w)
    raises("H has shape", oz.ozaki25_rms_norm_backward, X, X[:2], w)
    raises("dH must be", oz.ozaki25_rms_norm_backward, X, X, w, dH=X.float())
    raises("dweight must be", oz.ozaki25_rms_norm_backward, X, X, w, dweight=w)
    raises("workspace must be", oz.ozaki25_rms_norm_backward, X, X, w, workspace=w)
    raises("must be a CUDA tensor", oz.ozaki25_rms_norm_backward, X, X, w)


def test_binding_quantise():
    X = torch.zeros(4, 20)
    raises("2-D or 3-D", oz.ozaki25_quantise, X[0])
    raises("X must be a 2-D tensor of dtype", oz.ozaki25_quantise, X.double())
    raises("layout must be", oz.ozaki25_quantise, X, layout="cols")
    raises("X must be a CUDA tensor", oz.ozaki25_quantise, X)


def test_gradients_are_not_recorded():
    X, w = torch.zeros(4, 20, requires_grad=True), torch.ones(20)
    for call in (lambda: oz.ozaki25_rms_norm(X, w), lambda: oz.ozaki25_quantise(X), lambda: oz.ozaki25_rms_norm_backward(X, X, w)):
        with pytest.warns(UserWarning, match="does not record gradients"), pytest.raises(ValueError, match="CUDA"):
            call()
