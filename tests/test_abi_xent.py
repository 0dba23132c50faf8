"""Refusals of gc_softmax_xent before any launch (no GPU here)."""
import ctypes

import pytest
import torch

Q = ctypes.c_void_p(4096)


def _lib():
    return pytest.importorskip("paper_2405_19509_gb300", reason="libgc.so not built")


def _call(X=Q, ldx=64, xt=1, W=Q, ldw=64, wt=1, y=Q, N=2, n_c=3, C=64, V=100, loss=None, row_loss=Q, dX=Q, lddx=64,
          G=Q, ldg=6400, ws=Q, n=1 << 40):
    return _lib().lib.gc_softmax_xent(X, ldx, xt, W, ldw, wt, y, 1, N, n_c, C, V, loss, row_loss, None, dX, lddx, G,
                                      ldg, ws, n, None)


@pytest.mark.parametrize("kw,code", [
    (dict(X=None), -1), (dict(W=None), -1), (dict(y=None), -1), (dict(xt=2), -1), (dict(wt=-1), -1),
    (dict(row_loss=None, dX=None, G=None), -1), (dict(N=0), -2), (dict(n_c=0), -2), (dict(C=0), -2), (dict(V=0), -2),
    (dict(N=1 << 16, n_c=1 << 15), -3), (dict(C=(1 << 20) + 1), -3), (dict(V=(1 << 28) + 1), -3),
    (dict(N=1, n_c=1 << 30, V=1 << 20), -3), (dict(ldx=63), -2), (dict(ldw=63), -2), (dict(lddx=63), -2),
    (dict(ldg=6399), -2), (dict(y=ctypes.c_void_p(4100)), -1), (dict(G=ctypes.c_void_p(4098)), -1),
    (dict(ws=None), -6), (dict(n=1000), -6), (dict(ws=ctypes.c_void_p(4160)), -6)])
def test_refusals(kw, code):
    assert _call(**kw) == code


def test_workspace_keeps_no_logits():
    """Of 65,536 points and 65,536 columns the logits would be 17 GB in fp32: the scratch holds a piece."""
    L = _lib().lib
    full = L.gc_softmax_xent_workspace(64, 1024, 512, 65536, 1, 1, 1, 3)
    score = L.gc_softmax_xent_workspace(64, 1024, 512, 65536, 1, 1, 1, 0)
    assert 0 < score < full < 1 << 30
    assert L.gc_softmax_xent_workspace(0, 1, 1, 1, 1, 1, 1, 0) == 0
    # rows off the 16-byte boundaries are copied
    assert L.gc_softmax_xent_workspace(1, 9, 512, 65536, 1, 1, 0, 0) >= 65536 * 1024


def test_binding_checks():
    gc = _lib()
    X, W = torch.zeros(6, 8), torch.zeros(5, 8)
    with pytest.raises(ValueError):
        gc.gc_softmax_xent(X, W, torch.zeros(6, dtype=torch.long), 2, 4)
    with pytest.raises(TypeError):
        gc.gc_softmax_xent(X, W, torch.zeros(6), 2, 3)
    with pytest.raises(TypeError):
        gc.gc_softmax_xent(X, W, torch.zeros(6, dtype=torch.long), 2, 3)   # not on the GPU


def test_no_copy_goes_to_another_sm():
    """The library also runs in programs of several GPUs: no TMA copy in its sources names more than one CTA."""
    import glob
    import os
    import re
    csrc = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2405_19509_gb300", "csrc")
    files = sorted(glob.glob(os.path.join(csrc, "*.cu*")))
    assert files
    for f in files:
        with open(f) as h:
            text = re.sub(r'"\s*"', "", h.read())       # neighbouring string literals are one
        assert not re.search(r"cp\.async\.bulk[\w.:]*multicast", text), os.path.basename(f)
