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
