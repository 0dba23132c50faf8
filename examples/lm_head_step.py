"""Coded training of a language model's output end under partial stragglers.

The parameters are one vector w = [gamma, beta, W]: the last layer norm and the output matrix over the
vocabulary.  An iteration does what the workers and the parameter server would:

  forward   y, h = layer norm of (residual + dropout(branch)); losses over the vocabulary
  backward  gradients per chunk, in the layout the code takes: G[i] = [dgamma, dbeta, dW] of chunk i;
            and of the branch and the residual, for the layers below
  code      coefficients for the chunks that were finished (Algorithm 1), encode, decode and update

The dropout mask is a function of (seed, iteration, point, column), so the workers that hold a chunk
agree on its gradient, up to the order of sums: worker_gradient() is what one of them computes from its
own rows.

    python examples/lm_head_step.py [iterations]
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
    """Synthetic activations and labels: tokens whose branch points at their label's direction."""

    def __init__(self, N=6, n_c=128, C=256, V=1000, delta=3, ell=2, p=0.1, seed=0, device="cuda",
                 dtype=torch.bfloat16):
        self.N, self.n_c, self.C, self.V, self.delta, self.ell, self.p, self.seed = N, n_c, C, V, delta, ell, p, seed
        g = torch.Generator(device=device).manual_seed(seed)
        T = N * n_c
        self.y = torch.randint(0, V, (T,), generator=g, device=device)
        self.y[::17] = -100                                            # padding
        direction = torch.randn(V, C, generator=g, device=device)
        self.branch = (direction[self.y.clamp_min(0)] + 0.5 * torch.randn(T, C, generator=g, device=device)).to(dtype)
        self.residual = (0.5 * torch.randn(T, C, generator=g, device=device)).to(dtype)
        self.w = torch.cat([torch.ones(C, device=device), torch.zeros(C, device=device),
                            torch.randn(V * C, generator=g, device=device) / C ** 0.5])
        _, order, _ = gc.gc_make_assignment(N, N, delta, gc.GC_CYCLIC)
        rng = np.random.default_rng(seed)
        self.R = torch.from_numpy(rng.standard_normal((ell, N))).to(device)   # the server's Gaussian matrix
        self.order = torch.from_numpy(order).to(device)
        self.rng = rng
        self.ws = gc.Workspace(device)

    @property
    def d(self):
        return 2 * self.C + self.V * self.C

    def slices(self, w):
        C = self.C
        return w[:C], w[C:2 * C], w[2 * C:].view(self.V, C)


def gradients(pb: Problem, step: int, rows=slice(None), chunks=None, G=None):
    """Mean loss, chunk gradients (chunks x d) and the gradients that go down to branch and residual, of
    the points `rows` (whole chunks)."""
    chunks = pb.N if chunks is None else chunks
    branch, residual, y = pb.branch[rows], pb.residual[rows], pb.y[rows]
    first = rows.start or 0
    gamma, beta, W = pb.slices(pb.w)
    drop = dict(p=pb.p, seed=pb.seed, offset=step, row0=first)
    if G is None:
        G = torch.empty(chunks, pb.d, device=branch.device)
    f = gc.gc_layer_norm(branch, gamma, beta, residual=residual, **drop)
    head = gc.gc_softmax_xent(f["y"], W, y, chunks, pb.n_c, G=G[:, 2 * pb.C:], ws=pb.ws)
    back = gc.gc_layer_norm_backward(head["dX"], f["h"], f["mean"], f["rstd"], gamma, chunks, pb.n_c,
                                     dresidual=True, G=G[:, :2 * pb.C], ws=pb.ws, **drop)
    return head["loss"], G, back["dx"], back["dresidual"]


def worker_gradient(pb: Problem, step: int, chunk: int):
    """What any worker that holds `chunk` computes for it, from that chunk's rows alone."""
    rows = slice(chunk * pb.n_c, (chunk + 1) * pb.n_c)
    return gradients(pb, step, rows, 1)[1][0]


def train(pb: Problem, iterations: int, lr: float = 2.0):
    """Losses of coded gradient descent; every iteration each worker has finished some of its chunks."""
    losses = []
    G = torch.empty(pb.N, pb.d, device=pb.w.device)
    for step in range(iterations):
        loss, G, _, _ = gradients(pb, step, G=G)
        psi = torch.from_numpy(pb.rng.integers(1, pb.delta + 1, (1, pb.N)).astype(np.int32)).to(pb.w.device)
        E = gc.gc_find_encoding_coeff(pb.R, pb.ell, pb.order, pb.N, pb.N, pb.delta, psi, C=False, delta_out=False,
                                      coef_err=False, est=False, ws=pb.ws)["E"]
        gc.gc_live_step(E, pb.R, pb.ell, pb.order, pb.N, pb.N, pb.delta, psi, G, pb.w, lr, pb.N * pb.n_c)
        losses.append(loss)
    gc.gc_status(pb.ws)
    return [v.item() for v in losses]


if __name__ == "__main__":
    n = int(sys.argv[1]) if len(sys.argv) > 1 else 40
    pb = Problem()
    whole = gradients(pb, 0)[1][2]
    off = (worker_gradient(pb, 0, 2) - whole).abs().max() / whole.abs().max()
    losses = train(pb, n)
    print(f"a worker's gradient of its chunk against that of all chunks together: {off.item():.1e} of the largest")
    print("loss " + " ".join(f"{v:.3f}" for v in losses[:: max(1, n // 10)]) + f" -> {losses[-1]:.3f}")
