"""Refusals of gc_orthogonalize and gc_muon_step before any launch (no GPU here)."""
import ctypes

import pytest
import torch

Q, P, S = (ctypes.c_void_p(4096 * i) for i in (1, 2, 3))
BAD4, BAD2 = ctypes.c_void_p(4098), ctypes.c_void_p(4097)


def _lib():
    return pytest.importorskip("paper_2405_19509_gb300", reason="libgc.so not built")


def _c(*v):
    return (ctypes.c_float * 3)(*v)


def _ortho(U=Q, ldu=64, su=6400, dt=0, batch=2, rows=100, cols=64, co=None, steps=5, eps=1e-7, out=P, ldo=64, so=6400, ws=Q,
           n=1 << 40):
    return _lib().lib.gc_orthogonalize(U, ldu, su, dt, batch, rows, cols, co, steps, eps, out, ldo, so, ws, n, None)


def _muon(w=Q, ldw=64, sw=6400, m=P, ldm=64, sm=6400, g=S, ldg=64, sg=6400, batch=2, rows=100, cols=64, lr=0.1, Ntil=7, mu=0.9,
          nest=1, wd=0.0, scale=1.0, co=None, steps=5, eps=1e-7, ws=Q, n=1 << 40):
    return _lib().lib.gc_muon_step(w, ldw, sw, m, ldm, sm, g, ldg, sg, batch, rows, cols, lr, Ntil, mu, nest, wd, scale, co, steps,
                                   eps, ws, n, None)


COMMON = [
    (dict(batch=-1), -2), (dict(rows=0), -2), (dict(cols=0), -2), (dict(rows=(1 << 20) + 1), -3),
    (dict(rows=(1 << 15) + 1, cols=(1 << 15) + 1), -3), (dict(batch=(1 << 20) + 1), -3),
    (dict(batch=1 << 20, rows=1 << 11, cols=1 << 11), -3), (dict(steps=0), -1), (dict(steps=65), -1), (dict(eps=-1.0), -1),
    (dict(eps=float("nan")), -1), (dict(eps=float("inf")), -1), (dict(co=_c(3.4445, 4.775, 2.0315)), -1),
    (dict(co=_c(float("nan"), 0, 0)), -1), (dict(co=_c(1.5, -0.5, float("inf"))), -1), (dict(co=_c(100, -200, 100)), -1),
    (dict(co=_c(4.5, 0, 0)), -1), (dict(ws=None), -6), (dict(n=255), -6), (dict(ws=ctypes.c_void_p(4160)), -6),
]


@pytest.mark.parametrize("kw,code", COMMON + [
    (dict(U=None), -1), (dict(out=None), -1), (dict(dt=2), -1), (dict(dt=-1), -1), (dict(U=BAD4), -1), (dict(out=BAD2, dt=1), -1),
    (dict(ldu=63), -2), (dict(ldo=63), -2), (dict(su=6399), -2), (dict(so=6399), -2), (dict(so=0), -2), (dict(so=-6400), -2),
    (dict(ldu=127, su=64), -2), (dict(ldu=128, su=63), -2)])
def test_orthogonalize_refusals(kw, code):
    assert _ortho(**kw) == code


@pytest.mark.parametrize("kw,code", COMMON + [
    (dict(w=None), -1), (dict(m=None), -1), (dict(g=None), -1), (dict(Ntil=0), -1), (dict(w=BAD4), -1), (dict(m=BAD4), -1),
    (dict(g=BAD4), -1), (dict(w=P), -1), (dict(g=Q), -1), (dict(g=P), -1), (dict(ldw=63), -2), (dict(ldm=63), -2),
    (dict(ldg=63), -2), (dict(sw=6399), -2), (dict(sm=6399), -2), (dict(sg=6399), -2)])
def test_muon_refusals(kw, code):
    assert _muon(**kw) == code


def test_an_empty_batch_launches_nothing():
    assert _ortho(batch=0, U=None) == 0 and _muon(batch=0, w=None) == 0


@pytest.mark.parametrize("co", [None, _c(3.4445, -4.7750, 2.0315), _c(1.875, -1.25, 0.375), _c(1.5, -0.5, 0), _c(2, -1.5, 0.5), _c(0, 0, 0)])
def test_coefficients_that_are_taken(co):
    """They pass to the next check, the workspace's."""
    assert _ortho(co=co, steps=64, n=0) == -6


def test_workspace():
    f = _lib().lib.gc_orthogonalize_workspace
    assert f(1, 100, 64, 2) == 0 and f(-1, 1, 1, 0) == 0 and f(1, 0, 1, 0) == 0 and f(0, 5, 5, 0) == 256
    m, n = 2048, 8192
    assert 8 * m * n + 8 * m * m <= f(1, m, n, 0) < 1.5 * (8 * m * n + 8 * m * m)
    assert f(1, n, m, 0) == f(1, m, n, 0) and f(3, 100, 64, 1) <= f(3, 100, 64, 0)


def test_binding_checks():
    gc = _lib()
    a = torch.zeros(6, 8)
    for bad in (a, a.half(), a[0], None):
        with pytest.raises(TypeError):
            gc.gc_orthogonalize(bad)
    with pytest.raises(TypeError):
        gc.gc_muon_step(a, a.clone(), a.clone(), 0.1, 1)
