"""Coded training of a language model's last block, whose matrices are updated by orthogonalised momentum.

The parameters are one vector w = [gamma, beta, W1, b1, W2, b2, V]: the block's layer norm, its two matrices with their
biases, and the output matrix over the vocabulary.  An iteration does what the workers and the parameter server would:

  forward   n = layer norm of x; a = gelu(n W1^T + b1); h = x + a W2^T + b2; losses of h over the vocabulary
  backward  gradients per chunk, in the layout the code takes: G[i] = [dgamma, dbeta, dW1, db1, dW2, db2, dV] of chunk i;
            and of x, for the layers below
  code      coefficients for the chunks that were finished (Algorithm 1), encode, decode
  update    W1 and W2 by gc_muon_step, the vectors and the output matrix by gc_sgd_step, each on its slice of w and of the
            decoded gradient

    python examples/lm_block_step.py [iterations]
"""
from __future__ import annotations

import os
import sys

import numpy as np
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import paper_2405_19509_gb300 as gc  # noqa: E402


class Problem:
    """Synthetic activations and labels: a label is where a random matrix takes the activation."""

    def __init__(self, N=6, n_c=128, C=256, F=1024, V=1000, delta=3, ell=2, seed=0, device="cuda", dtype=torch.bfloat16):
        self.N, self.n_c, self.C, self.F, self.V, self.delta, self.ell = N, n_c, C, F, V, delta, ell
        g = torch.Generator(device=device).manual_seed(seed)

        def randn(*shape):
            return torch.randn(*shape, generator=g, device=device)
        T = N * n_c
        self.x = randn(T, C).to(dtype)
        self.y = (self.x.float() @ randn(C, V)).argmax(1)
        self.y[::17] = -100                                            # padding
        shapes = dict(gamma=(C,), beta=(C,), W1=(F, C), b1=(F,), W2=(C, F), b2=(C,), V=(V, C))
        start = dict(gamma=torch.ones(C, device=device), W1=randn(F, C) / C ** 0.5, W2=0.1 * randn(C, F) / F ** 0.5,
                     V=randn(V, C) / C ** 0.5)
        self.shapes, self.at, n = shapes, {}, 0
        for k, s in shapes.items():
            self.at[k] = slice(n, n + int(np.prod(s)))
            n = self.at[k].stop
        self.d = n
        self.w = torch.zeros(n, device=device)
        for k, v in start.items():
            self.w[self.at[k]] = v.flatten()
        self.momentum = {k: torch.zeros(shapes[k], device=device) for k in ("W1", "W2")}
        _, order, _ = gc.gc_make_assignment(N, N, delta, gc.GC_CYCLIC)
        self.rng = np.random.default_rng(seed)
        self.R = torch.from_numpy(self.rng.standard_normal((ell, N))).to(device)   # the server's Gaussian matrix
        self.order = torch.from_numpy(order).to(device)
        self.ws = gc.Workspace(device)

    def slices(self, w):
        return {k: w[self.at[k]].view(s) for k, s in self.shapes.items()}


def gradients(pb: Problem, rows=slice(None), chunks=None, G=None):
    """Mean loss, chunk gradients (chunks x d) and the gradient of x, of the points `rows` (whole chunks)."""
    chunks = pb.N if chunks is None else chunks
    x, y = pb.x[rows], pb.y[rows]
    p, n_c, ws = pb.slices(pb.w), pb.n_c, pb.ws
    if G is None:
        G = torch.empty(chunks, pb.d, device=x.device)

    def at(k):
        return G[:, pb.at[k]]
    f = gc.gc_layer_norm(x, p["gamma"], p["beta"])
    a = gc.gc_linear(f["y"], p["W1"], p["b1"], gc.GC_ACT_GELU, z=True, ws=ws)
    h = gc.gc_linear(a["y"], p["W2"], p["b2"], residual=x, ws=ws)["y"]
    head = gc.gc_softmax_xent(h, p["V"], y, chunks, n_c, G=at("V"), ws=ws)
    da = gc.gc_linear_backward(head["dX"], a["y"], p["W2"], chunks, n_c, G=at("W2"), Gb=at("b2"), ws=ws)["dx"]
    dn = gc.gc_linear_backward(da, f["y"], p["W1"], chunks, n_c, z=a["z"], act=gc.GC_ACT_GELU, G=at("W1"), Gb=at("b1"),
                               ws=ws)["dx"]
    # dX of the head is also the gradient of the block's residual: it joins that of the layer norm
    norm = G[:, pb.at["gamma"].start:pb.at["beta"].stop]
    back = gc.gc_layer_norm_backward(dn, f["h"], f["mean"], f["rstd"], p["gamma"], chunks, n_c, dh=head["dX"], G=norm, ws=ws)
    return head["loss"], G, back["dx"]


def worker_gradient(pb: Problem, chunk: int):
    """What any worker that holds `chunk` computes for it, from that chunk's rows alone."""
    return gradients(pb, slice(chunk * pb.n_c, (chunk + 1) * pb.n_c), 1)[1][0]


def decoded(pb: Problem, G, psi):
    """The decoded gradient (d) of the pattern psi (1 x m processed counts)."""
    T = gc.gc_encode(pb.R, pb.ell, pb.order, pb.N, pb.N, pb.delta, psi, G, ws=pb.ws)
    return gc.gc_decode_tx(pb.R, pb.ell, pb.N, T, pb.d)[0]


def update(pb: Problem, g, lr: float, lr_matrix: float):
    """w after a step along the decoded gradient g, a sum over all points."""
    points = pb.N * pb.n_c
    for k, at in pb.at.items():
        if k in pb.momentum:
            shape = pb.shapes[k]
            gc.gc_muon_step(pb.w[at].view(shape), pb.momentum[k], g[at].view(shape), lr_matrix, points,
                            scale=0.2 * max(shape) ** 0.5, ws=pb.ws)
        else:
            gc.gc_sgd_step(pb.w[at], g[at], lr, points)


def train(pb: Problem, iterations: int, lr: float = 0.1, lr_matrix: float = 0.005):
    """Losses of coded training; every iteration each worker has finished some of its chunks."""
    losses = []
    G = torch.empty(pb.N, pb.d, device=pb.w.device)
    for _ in range(iterations):
        loss, G, _ = gradients(pb, G=G)
        psi = torch.from_numpy(pb.rng.integers(1, pb.delta + 1, (1, pb.N)).astype(np.int32)).to(pb.w.device)
        update(pb, decoded(pb, G, psi), lr, lr_matrix)
        losses.append(loss)
    gc.gc_status(pb.ws)
    return [v.item() for v in losses]


if __name__ == "__main__":
    n = int(sys.argv[1]) if len(sys.argv) > 1 else 40
    pb = Problem()
    whole = gradients(pb)[1][2]
    off = (worker_gradient(pb, 2) - whole).abs().max() / whole.abs().max()
    losses = train(pb, n)
    print(f"a worker's gradient of its chunk against that of all chunks together: {off.item():.1e} of the largest")
    print("loss " + " ".join(f"{v:.3f}" for v in losses[:: max(1, n // 10)]) + f" -> {losses[-1]:.3f}")
