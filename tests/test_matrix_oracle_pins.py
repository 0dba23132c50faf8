"""Pins of the fp64 oracle's linear layers and orthogonalised updates (CPU): every gradient against central differences, the
products against their singular values."""
import numpy as np
import pytest

from oracle import lm_oracle as L


def _differences(f, x, step=1e-5):
    g = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        a, b = x.copy(), x.copy()
        a[i] += step
        b[i] -= step
        g[i] = (f(a) - f(b)) / (2 * step)
    return g


@pytest.mark.parametrize("act", ["none", "relu", "gelu", "gelu_tanh", "silu"])
def test_linear_gradient_against_differences(act):
    """Step 1e-5: the cubic term is 1e-10, rounding 1e-11 of values of order 1; relu has no kink within a step."""
    rng = np.random.default_rng(2)
    N, n_c, C, F = 2, 3, 4, 5
    x, W, b, dy = (rng.standard_normal(s) for s in ((N * n_c, C), (F, C), F, (N * n_c, F)))
    y, z = L.linear(x, W, b, act, residual=dy)
    assert np.abs(z).min() > 1e-3 and np.allclose(y - dy, L.linear(x, W, b, act)[0])
    dx, G, Gb = L.linear_grad(dy, z, x, W, act, N)
    total = lambda x, W, b, r=slice(None): (L.linear(x, W, b, act)[0] * dy)[r].sum()
    assert np.allclose(dx, _differences(lambda t: total(t, W, b), x), atol=1e-8)
    for i in range(N):
        r = slice(i * n_c, (i + 1) * n_c)
        assert np.allclose(G[i].reshape(F, C), _differences(lambda t: total(x, t, b, r), W), atol=1e-8)
        assert np.allclose(Gb[i], _differences(lambda t: total(x, W, t, r), b), atol=1e-8)


def test_gelu_by_its_tanh():
    """The cubic's tanh is within 1e-3 of the error function's form (published with it)."""
    z = np.linspace(-8, 8, 1001)
    assert np.abs(L.activation(z, "gelu") - L.activation(z, "gelu_tanh")).max() < 1e-3


@pytest.mark.parametrize("rows,cols", [(4, 9), (9, 4), (5, 5), (1, 7), (7, 1)])
def test_orthogonalize_by_singular_values(rows, cols):
    """The steps act on each singular value alone, as a scalar polynomial; the vectors stay."""
    u = np.random.default_rng(rows).standard_normal((rows, cols))
    p, s, q = np.linalg.svd(u, full_matrices=False)
    a, b, c = 3.4445, -4.7750, 2.0315
    s = s / np.sqrt((s ** 2).sum())
    for _ in range(5):
        s = a * s + b * s ** 3 + c * s ** 5
    assert np.allclose(L.orthogonalize(u), (p * s) @ q)
    assert np.allclose(L.orthogonalize(u.T), L.orthogonalize(u).T)
    assert not L.orthogonalize(np.zeros((rows, cols))).any()


def test_orthogonalize_converges_with_the_classical_coefficients():
    """(15, -10, 3) / 8, whose fixed point is 1: an orthogonal matrix after enough steps."""
    u = np.random.default_rng(4).standard_normal((4, 9))
    o = L.orthogonalize(u, (1.875, -1.25, 0.375), 30)
    assert np.allclose(o @ o.T, np.eye(4))


def test_muon_step():
    rng = np.random.default_rng(5)
    w, m, g = (rng.standard_normal((3, 5)) for _ in range(3))
    w1, m1 = L.muon_step(w, m, g, 0.1, 4, mu=0.9, nesterov=False, weight_decay=0.5, scale=2.0)
    assert np.allclose(m1, 0.9 * m + g / 4) and np.allclose(w1, 0.95 * w - 0.2 * L.orthogonalize(m1))
    w2, m2 = L.muon_step(w, m, g, 0.1, 4, mu=0.9)
    assert np.allclose(m2, m1) and np.allclose(w2, w - 0.1 * L.orthogonalize(g / 4 + 0.9 * m1))
