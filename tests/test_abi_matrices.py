"""Refusals of linear layers and orthogonalised matrices, of outputs over inputs and of more blocks than a launch has (no GPU here)."""
import ctypes

import pytest

from test_abi_linear import P, Q, _bwd, _fwd, _lib
from test_abi_muon import _ortho


@pytest.mark.parametrize("kw", [dict(y=P), dict(z=P)])
def test_outputs_over_the_weights(kw):
    assert _fwd(**kw) == -1


@pytest.mark.parametrize("kw,code", [
    (dict(ldo=72, so=7200), -1), (dict(so=6464), -1), (dict(ldo=128, so=64), -1),            # a matrix's result over the next one's input
    (dict(), -6), (dict(batch=1, ldo=72), -6), (dict(batch=1, so=1), -6), (dict(rows=1, ldo=99), -6)])
def test_a_batch_over_itself_in_another_layout(kw, code):
    assert _ortho(**{**dict(out=Q, n=0), **kw}) == code


@pytest.mark.parametrize("kw", [dict(F=1, C=33), dict(F=1, C=33, dX=None, W=None), dict(F=1, C=33, Gb=None)])
def test_more_blocks_than_a_launch_has(kw):
    """2^30 chunks of a point and two tiles of G each; the same sizes without G are refused for nothing."""
    size = dict(N=1 << 30, n_c=1, lddy=64, ldz=64, ldgb=64, n=0)
    assert _bwd(**{**size, **kw}) == -3
    assert _bwd(**{**size, **kw, "dX": ctypes.c_void_p(1 << 40), "W": P, "G": None}) == -6
    f = _lib().lib.gc_linear_backward_workspace
    assert f(1 << 30, 1, kw["C"], kw["F"], 1, 1, 2, 1, 1, 1, 3) == 0 and f(1 << 30, 1, kw["C"], kw["F"], 1, 1, 2, 1, 1, 1, 1) > 0


def test_as_many_blocks_as_a_launch_has():
    assert _bwd(N=(1 << 30) - (1 << 27), n_c=1, F=1, C=33, lddy=64, ldz=64, ldgb=64, n=0) == -6


def test_version():
    """0.4: the linear layers and the orthogonalised matrices."""
    assert _lib().gc_version() >= 400
