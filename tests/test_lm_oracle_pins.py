"""Pins of the fp64 oracle of the language-model operators (CPU): published vectors of the generator,
and every gradient against central differences of the function it is the gradient of."""
import numpy as np
import pytest

from oracle import lm_oracle as L

# Known answers published with the generator (counter, key -> words).
KAT = [
    ((0, 0, 0, 0), (0, 0), (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
    ((0xFFFFFFFF,) * 4, (0xFFFFFFFF,) * 2, (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
    ((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0),
     (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1)),
]


@pytest.mark.parametrize("counter,key,words", KAT)
def test_philox_known_answers(counter, key, words):
    assert tuple(L.philox4x32_10(counter, key)) == words


def test_mask_is_a_function_of_the_point():
    """Any rows of a matrix draw what the whole matrix draws for them; other numbers draw others."""
    a = L.keep_mask(9, 21, 0.4, 77, 5)
    assert np.array_equal(L.keep_mask(4, 21, 0.4, 77, 5, row0=3), a[3:7])
    assert not np.array_equal(L.keep_mask(9, 21, 0.4, 78, 5), a)
    assert not np.array_equal(L.keep_mask(9, 21, 0.4, 77, 6), a)


def test_mask_rate_and_unbiased_scale():
    """Of 64 x 1024 numbers the share kept is within 5 standard deviations of 1 - t / 2^16, and the
    scale is its inverse."""
    p, n = 0.3, 64 * 1024
    q = 1 - L.drop_threshold(p) / 65536
    k = L.keep_mask(64, 1024, p, 3, 1)
    assert abs(k.mean() - q) <= 5 * np.sqrt(q * (1 - q) / n)
    out = L.dropout(np.ones((64, 1024)), p, 3, 1)
    assert np.allclose(out[k], 1 / q) and not out[~k].any()


def _differences(f, x, step=1e-5):
    """Central differences of the scalar f at every element of x."""
    g = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        a, b = x.copy(), x.copy()
        a[i] += step
        b[i] -= step
        g[i] = (f(a) - f(b)) / (2 * step)
    return g


def test_layer_norm_gradient_against_differences():
    rng = np.random.default_rng(1)
    N, n_c, C, eps, p = 2, 3, 5, 1e-3, 0.25
    x, r, dy = (rng.standard_normal((N * n_c, C)) for _ in range(3))
    gamma, beta = 1 + 0.3 * rng.standard_normal(C), rng.standard_normal(C)

    def total(x, r, gamma, beta, rows=slice(None)):
        h = L.dropout(x, p, 9, 2, residual=r)
        return (L.layer_norm(h, gamma, beta, eps)[0] * dy)[rows].sum()
    h = L.dropout(x, p, 9, 2, residual=r)
    _, mean, rstd = L.layer_norm(h, gamma, beta, eps)
    d, G = L.layer_norm_grad(dy, h, mean, rstd, gamma, N)
    # the third derivative's part of a central difference is about 1e-9 here
    assert np.allclose(_differences(lambda v: total(x, v, gamma, beta), r), d, atol=1e-7)
    assert np.allclose(_differences(lambda v: total(v, r, gamma, beta), x), L.dropout(d, p, 9, 2), atol=1e-7)
    for i in range(N):
        rows = slice(i * n_c, (i + 1) * n_c)
        assert np.allclose(_differences(lambda v: total(x, r, v, beta, rows), gamma), G[i, :C], atol=1e-7)
        assert np.allclose(_differences(lambda v: total(x, r, gamma, v, rows), beta), G[i, C:], atol=1e-7)


def test_softmax_xent_gradient_against_differences():
    rng = np.random.default_rng(2)
    N, n_c, C, V = 2, 3, 4, 7
    X, W = rng.standard_normal((N * n_c, C)), rng.standard_normal((V, C))
    y = np.array([0, 6, -100, 3, 3, -1])
    loss, lse, dX, G = L.softmax_xent(X, W, y, N)
    assert loss[2] == 0 and loss[5] == 0 and not dX[2].any()
    assert np.allclose(loss[0], -np.log(np.exp(X[0] @ W[0]) / np.exp(X[0] @ W.T).sum()))
    assert np.allclose(_differences(lambda v: L.softmax_xent(v, W, y, N)[0].sum(), X), dX, atol=1e-7)
    for i in range(N):
        f = lambda v: L.softmax_xent(X, v, y, N)[0][i * n_c:(i + 1) * n_c].sum()
        assert np.allclose(_differences(f, W), G[i], atol=1e-7)


def test_softmax_xent_of_one_class_is_zero():
    loss, lse, dX, G = L.softmax_xent(np.ones((2, 3)), np.ones((1, 3)), np.array([0, 0]), 1)
    assert not loss.any() and not dX.any() and not G.any()
