"""Refusals of linear layers and orthogonalised matrices, of outputs over inputs and of more blocks than a launch has (no GPU here)."""
import ctypes

import pytest

from test_abi_linear import P, Q, _bwd, _fwd, _lib


@pytest.mark.parametrize("kw", [dict(y=P), dict(z=P)])
def test_outputs_over_the_weights(kw):
    assert _fwd(**kw) == -1
