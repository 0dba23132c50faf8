"""Refusals of gc_linear and gc_linear_backward before any launch (no GPU here)."""
import ctypes

import pytest
import torch

Q, P, S, U = (ctypes.c_void_p(4096 * i) for i in (1, 2, 3, 4))
BAD4, BAD2 = ctypes.c_void_p(4098), ctypes.c_void_p(4097)


def _lib():
    return pytest.importorskip("paper_2405_19509_gb300", reason="libgc.so not built")


def _fwd(X=Q, ldx=64, xt=1, W=P, ldw=64, wt=1, bias=None, act=0, res=None, ldr=100, rows=6, C=64, F=100, y=S, ldy=100,
         z=None, ldz=100, ws=Q, n=1 << 40):
    return _lib().lib.gc_linear(X, ldx, xt, W, ldw, wt, bias, act, res, ldr, rows, C, F, y, ldy, z, ldz, ws, n, None)


@pytest.mark.parametrize("kw,code", [
    (dict(X=None), -1), (dict(W=None), -1), (dict(y=None), -1), (dict(xt=2), -1), (dict(wt=-1), -1), (dict(act=5), -1),
    (dict(act=-1), -1), (dict(rows=-1), -2), (dict(C=0), -2), (dict(F=0), -2), (dict(rows=(1 << 30) + 1), -3),
    (dict(C=(1 << 20) + 1), -3), (dict(F=(1 << 20) + 1), -3), (dict(rows=1 << 30, F=1 << 20), -3), (dict(ldx=63), -2),
    (dict(ldw=63), -2), (dict(ldy=99), -2), (dict(z=U, ldz=99), -2), (dict(res=U, ldr=99), -2), (dict(bias=BAD4), -1),
    (dict(X=BAD2), -1), (dict(y=BAD2), -1), (dict(X=BAD4, xt=0), -1), (dict(y=Q), -1), (dict(z=Q), -1), (dict(z=S), -1),
    (dict(z=U, res=U), -1), (dict(res=S, ldr=104), -1), (dict(ws=None), -6), (dict(n=255), -6), (dict(ws=ctypes.c_void_p(4160)), -6),
    (dict(wt=0, rows=100000, n=4096), -6)])
def test_forward_refusals(kw, code):
    assert _fwd(**kw) == code


def test_no_rows_launch_nothing():
    assert _fwd(rows=0, X=None, y=None) == 0


def _bwd(dy=Q, lddy=100, z=U, ldz=100, X=Q, ldx=64, xt=1, W=P, ldw=64, wt=1, act=2, N=2, n_c=3, C=64, F=100, dX=S, lddx=64,
         G=S, ldg=6400, Gb=S, ldgb=100, ws=Q, n=1 << 40):
    return _lib().lib.gc_linear_backward(dy, lddy, z, ldz, X, ldx, xt, W, ldw, wt, act, N, n_c, C, F, dX, lddx, G, ldg, Gb,
                                         ldgb, ws, n, None)


@pytest.mark.parametrize("kw,code", [
    (dict(dy=None), -1), (dict(z=None), -1), (dict(X=None), -1), (dict(W=None), -1), (dict(dX=None, G=None, Gb=None), -1),
    (dict(xt=2), -1), (dict(wt=2), -1), (dict(act=5), -1), (dict(N=0), -2), (dict(n_c=0), -2), (dict(C=0), -2),
    (dict(F=0), -2), (dict(N=1 << 16, n_c=1 << 15), -3), (dict(C=(1 << 20) + 1), -3), (dict(F=(1 << 20) + 1), -3),
    (dict(N=1 << 20, n_c=1, C=1 << 17, F=1 << 17), -3), (dict(lddy=99), -2), (dict(ldz=99), -2), (dict(ldx=63), -2),
    (dict(ldw=63), -2), (dict(lddx=63), -2), (dict(ldg=6399), -2), (dict(ldgb=99), -2), (dict(G=BAD4), -1),
    (dict(Gb=BAD4), -1), (dict(dy=BAD2), -1), (dict(dX=Q), -1), (dict(dX=P), -1), (dict(dX=U), -1), (dict(ws=None), -6),
    (dict(n_c=100000, n=1000), -6), (dict(ws=ctypes.c_void_p(4160)), -6)])
def test_backward_refusals(kw, code):
    assert _bwd(**kw) == code


def test_workspaces():
    L = _lib().lib
    f, b = L.gc_linear_workspace, L.gc_linear_backward_workspace
    assert f(8192, 2048, 8192, 1, 1, 1, 1) == 256                           # bf16 rows are read where they lie
    assert f(8192, 2048, 8192, 1, 1, 0, 1) >= 8192 * 2048 * 2
    assert f(8192, 2048, 8192, 1, 0, 1, 1) >= 8192 * 2048 * 4               # an fp32 W as hi + lo
    assert f(8192, 2048, 8192, 0, 0, 1, 1) >= 2 * 8192 * 2048 * 6
    assert f(-1, 1, 1, 1, 1, 1, 1) == 0 and f(1, 0, 1, 1, 1, 1, 1) == 0 and f(0, 8, 8, 1, 1, 1, 1) == 256
    assert b(8, 1024, 2048, 8192, 1, 1, 0, 1, 1, 1, 3) == 256               # nor is dy copied without an activation
    assert b(8, 1024, 2048, 8192, 1, 1, 2, 1, 1, 1, 3) >= 8192 * 8192 * 4
    assert b(0, 1, 1, 1, 1, 1, 0, 1, 1, 1, 1) == 0


def test_binding_checks():
    gc = _lib()
    x, W = torch.zeros(6, 8), torch.zeros(5, 8)
    with pytest.raises(TypeError):
        gc.gc_linear(x, W)                                                  # not on the GPU
    with pytest.raises(TypeError):
        gc.gc_linear(x.half(), W)
    with pytest.raises(ValueError):
        gc.gc_linear_backward(torch.zeros(6, 5), x, W, 2, 4)
    with pytest.raises(TypeError):
        gc.gc_linear_backward(torch.zeros(6, 5), x, W, 2, 3)
