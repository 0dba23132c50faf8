"""fp64 oracle of the language-model operators: dropout by counters, layer norm and its gradient, and
softmax cross entropy over a vocabulary with its gradient, from their definitions.

Test infrastructure only; plain NumPy, no code shared with the CUDA path.
"""
from __future__ import annotations

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
