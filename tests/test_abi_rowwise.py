"""Refusals of gc_dropout, gc_layer_norm and gc_layer_norm_backward: codes returned by the C entry
points before any launch, and the binding's own checks (no GPU here)."""
import ctypes

import pytest
import torch


def _lib():
    return pytest.importorskip("paper_2405_19509_gb300", reason="libgc.so not built")


Q = ctypes.c_void_p(4096)
F = ctypes.c_float
D = ctypes.c_double


def _drop(x=Q, ldx=64, res=None, ldr=64, dtype=0, rows=4, cols=64, p=0.1, row0=0, out=Q, ldo=64):
    return _lib().lib.gc_dropout(x, ldx, res, ldr, dtype, rows, cols, p, 1, 2, row0, out, ldo, None)


def _norm(x=Q, dtype=0, rows=4, cols=64, eps=1e-5, p=0.0, y=Q, ldy=64, h=None):
    return _lib().lib.gc_layer_norm(x, 64, None, 0, dtype, rows, cols, None, None, eps, p, 1, 2, 0, y, ldy, h, 64,
                                    None, None, None)


def _grad(dy=Q, h=Q, mean=Q, rstd=Q, dtype=0, N=2, n_c=3, cols=64, p=0.0, dx=Q, dres=None, G=Q, ldg=128, ws=Q,
          n=1 << 30):
    return _lib().lib.gc_layer_norm_backward(dy, 64, h, 64, mean, rstd, None, None, 0, dtype, N, n_c, cols, p, 1,
                                             2, 0, dx, 64, dres, 64, G, ldg, ws, n, None)


@pytest.mark.parametrize("kw,code", [
    (dict(x=None), -1), (dict(out=None), -1), (dict(dtype=2), -1), (dict(p=1.0), -1), (dict(p=-0.1), -1),
    (dict(p=float("nan")), -1), (dict(rows=-1), -2), (dict(cols=0), -2), (dict(cols=32769), -3),
    (dict(ldx=63), -2), (dict(ldo=63), -2), (dict(res=Q, ldr=10), -2), (dict(row0=-1), -1),
    (dict(x=ctypes.c_void_p(4098)), -1), (dict(dtype=1, out=ctypes.c_void_p(4097)), -1),
    (dict(rows=0, x=None), 0)])
def test_dropout_refusals(kw, code):
    assert _drop(**kw) == code


@pytest.mark.parametrize("kw,code", [
    (dict(x=None), -1), (dict(y=None), -1), (dict(dtype=-1), -1), (dict(eps=-1.0), -1),
    (dict(eps=float("nan")), -1), (dict(p=1.5), -1), (dict(cols=40000), -3), (dict(rows=-2), -2),
    (dict(ldy=1), -2), (dict(h=ctypes.c_void_p(4099)), -1), (dict(rows=0), 0)])
def test_layer_norm_refusals(kw, code):
    assert _norm(**kw) == code


@pytest.mark.parametrize("kw,code", [
    (dict(dy=None), -1), (dict(h=None), -1), (dict(mean=None), -1), (dict(rstd=None), -1),
    (dict(dx=None, G=None), -1), (dict(N=0), -2), (dict(n_c=0), -2), (dict(N=1 << 16, n_c=1 << 16), -3),
    (dict(cols=32769), -3), (dict(ldg=127), -2), (dict(p=1.0), -1), (dict(ws=None), -6), (dict(n=10), -6),
    (dict(ws=ctypes.c_void_p(4104)), -6)])
def test_layer_norm_backward_refusals(kw, code):
    assert _grad(**kw) == code


def test_refusals_name_the_argument():
    gc = _lib()
    _drop(p=2.0)
    assert "p=2" in gc.gc_last_error()
    _grad(G=ctypes.c_void_p(4097))
    assert "G" in gc.gc_last_error()


def test_workspace_sizes():
    gc = _lib()
    assert gc.lib.gc_layer_norm_backward_workspace(0, 1, 1) == 0
    assert gc.lib.gc_layer_norm_backward_workspace(1, 1, 40000) == 0
    assert gc.lib.gc_layer_norm_backward_workspace(8, 2048, 4096) >= 256


def test_binding_checks():
    gc = _lib()
    x = torch.zeros(4, 8)
    with pytest.raises(TypeError):
        gc.gc_dropout(x, 0.1, 1)                     # not on the GPU
    with pytest.raises(TypeError):
        gc.gc_dropout(x.double(), 0.1, 1)
    with pytest.raises(TypeError):
        gc.gc_layer_norm(x[0])
    with pytest.raises(ValueError):
        gc.gc_layer_norm_backward(x, x, x[:, 0], x[:, 0], None, 3, 2)
