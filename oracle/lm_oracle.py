"""fp64 oracle of the language-model operators: dropout by counters, layer norm and its gradient,
softmax cross entropy over a vocabulary with its gradient, linear layers with theirs, and the orthogonalised
update of a matrix, from their definitions.

Test infrastructure only; plain NumPy, no code shared with the CUDA path.
"""
from __future__ import annotations

import math

import numpy as np

_M32 = 0xFFFFFFFF


def philox4x32_10(counter, key):
    """The four words of Philox4x32-10 (Salmon et al., SC 2011) at one counter (Python integers)."""
    x, k = list(counter), list(key)
    for _ in range(10):
        a, b = 0xD2511F53 * x[0], 0xCD9E8D57 * x[2]
        x = [(b >> 32) ^ x[1] ^ k[0], b & _M32, (a >> 32) ^ x[3] ^ k[1], a & _M32]
        k = [(k[0] + 0x9E3779B9) & _M32, (k[1] + 0xBB67AE85) & _M32]
    return x


def drop_threshold(p: float) -> int:
    """t: an element is dropped when its 16-bit number is below t."""
    return min(int(p * 65536 + 0.5), 65535)


def keep_mask(rows: int, cols: int, p: float, seed: int, offset: int, row0: int = 0) -> np.ndarray:
    """rows x cols booleans: element (r, c) is kept."""
    t = drop_threshold(p)
    groups = -(-cols // 8)
    out = np.zeros((rows, groups * 8), dtype=bool)
    for r in range(rows):
        for g in range(groups):
            e = (row0 + r) * groups + g
            w = philox4x32_10((e & _M32, e >> 32, offset & _M32, offset >> 32),
                              (seed & _M32, seed >> 32))
            for j in range(8):
                out[r, 8 * g + j] = ((w[j // 2] >> (16 * (j % 2))) & 0xFFFF) >= t
    return out[:, :cols]


def dropout(x, p, seed, offset, row0=0, residual=None):
    x = np.asarray(x, dtype=np.float64)
    if drop_threshold(p):
        keep = keep_mask(*x.shape, p, seed, offset, row0)
        x = np.where(keep, x * (65536 / (65536 - drop_threshold(p))), 0.0)
    return x if residual is None else x + np.asarray(residual, dtype=np.float64)


def layer_norm(h, gamma, beta, eps):
    """(y, mean, rstd) of the rows of h."""
    h = np.asarray(h, dtype=np.float64)
    mean = h.mean(1)
    rstd = 1 / np.sqrt(((h - mean[:, None]) ** 2).mean(1) + eps)
    return (h - mean[:, None]) * rstd[:, None] * gamma + beta, mean, rstd


def layer_norm_grad(dy, h, mean, rstd, gamma, N):
    """(gradient of h, G: N x 2 cols) for the gradient dy of y, chunks of equal rows."""
    dy, h = np.asarray(dy, dtype=np.float64), np.asarray(h, dtype=np.float64)
    mean, rstd = (np.asarray(v, dtype=np.float64)[:, None] for v in (mean, rstd))
    n = (h - mean) * rstd
    a = dy * gamma
    d = rstd * (a - a.mean(1, keepdims=True) - n * (a * n).mean(1, keepdims=True))
    rows = dy.shape[0] // N
    G = np.stack([np.concatenate([(dy[i * rows:(i + 1) * rows] * n[i * rows:(i + 1) * rows]).sum(0),
                                  dy[i * rows:(i + 1) * rows].sum(0)]) for i in range(N)])
    return d, G


def softmax_xent(X, W, y, N):
    """Per row the loss -log softmax(X W^T)[y] (0 where y < 0) and the log-sum-exp; the gradients of
    the summed loss: dX, and per chunk that of W (N x V x C).  Rows with y < 0 enter none of them."""
    X, W, y = np.asarray(X, dtype=np.float64), np.asarray(W, dtype=np.float64), np.asarray(y)
    live = y >= 0
    z = X @ W.T
    top = z.max(1)
    lse = top + np.log(np.exp(z - top[:, None]).sum(1))
    at = np.maximum(y, 0)
    loss = np.where(live, lse - z[np.arange(len(y)), at], 0.0)
    P = np.exp(z - lse[:, None])
    P[np.arange(len(y)), at] -= 1
    P[~live] = 0
    n_c = len(y) // N
    Xl = np.where(live[:, None], X, 0.0)
    G = np.stack([P[i * n_c:(i + 1) * n_c].T @ Xl[i * n_c:(i + 1) * n_c] for i in range(N)])
    return loss, lse, P @ W, G


_erf = np.vectorize(math.erf, otypes=[np.float64])


def activation(z, act):
    """act(z) of "none", "relu", "gelu", "gelu_tanh" or "silu"."""
    z = np.asarray(z, dtype=np.float64)
    if act == "relu":
        return np.maximum(z, 0)
    if act == "gelu":
        return 0.5 * z * (1 + _erf(z / math.sqrt(2)))
    if act == "gelu_tanh":
        return 0.5 * z * (1 + np.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))
    return z / (1 + np.exp(-z)) if act == "silu" else z


def activation_grad(z, act):
    """act'(z); of relu 0 at 0."""
    z = np.asarray(z, dtype=np.float64)
    if act == "relu":
        return (z > 0).astype(np.float64)
    if act == "gelu":
        return 0.5 * (1 + _erf(z / math.sqrt(2))) + z * np.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if act == "gelu_tanh":
        k = math.sqrt(2 / math.pi)
        t = np.tanh(k * (z + 0.044715 * z ** 3))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * k * (1 + 3 * 0.044715 * z * z)
    if act == "silu":
        s = 1 / (1 + np.exp(-z))
        return s * (1 + z * (1 - s))
    return np.ones_like(z)


def linear(x, W, bias=None, act="none", residual=None):
    """(y, z): z = x W^T + bias, y = residual + act(z)."""
    z = np.asarray(x, dtype=np.float64) @ np.asarray(W, dtype=np.float64).T
    if bias is not None:
        z = z + np.asarray(bias, dtype=np.float64)
    y = activation(z, act)
    return (y if residual is None else y + np.asarray(residual, dtype=np.float64)), z


def linear_grad(dy, z, x, W, act, N):
    """(dx, G: N x F C, Gb: N x F) for the gradient dy of y, chunks of equal rows."""
    d = np.asarray(dy, dtype=np.float64) * (1 if act == "none" else activation_grad(z, act))
    x = np.asarray(x, dtype=np.float64)
    parts = list(zip(np.split(d, N), np.split(x, N)))
    return (d @ np.asarray(W, dtype=np.float64), np.stack([(p.T @ q).ravel() for p, q in parts]),
            np.stack([p.sum(0) for p, _ in parts]))


def orthogonalize(u, coeffs=(3.4445, -4.7750, 2.0315), steps=5, eps=1e-7):
    """X <- (a + b X X^T + c (X X^T)^2) X, `steps` times, from u / max(|u|, eps) (Frobenius)."""
    u = np.asarray(u, dtype=np.float64)
    a, b, c = coeffs
    X = u / max(np.linalg.norm(u), eps)
    for _ in range(steps):
        A = X @ X.T
        X = a * X + (b * A + c * A @ A) @ X
    return X


def muon_step(w, momentum, g, lr, points, mu=0.95, nesterov=True, weight_decay=0.0, scale=1.0, **ns):
    """(w, momentum) after a step: momentum = mu momentum + g / points, and w = (1 - lr weight_decay) w
    - lr scale O, O the orthogonalised momentum (nesterov: g / points + mu times the new one)."""
    g = np.asarray(g, dtype=np.float64) / points
    m = mu * np.asarray(momentum, dtype=np.float64) + g
    o = orthogonalize(g + mu * m if nesterov else m, **ns)
    return (1 - lr * weight_decay) * np.asarray(w, dtype=np.float64) - lr * scale * o, m
