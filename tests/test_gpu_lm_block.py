"""Linear layers, layer norm, cross entropy, the code and the update by orthogonalised momentum together, as
examples/lm_block_step.py runs them."""
import os
import sys

import numpy as np
import pytest
import torch

import oracle as O
from oracle import lm_oracle as L
from _parity import rel_inf

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def ex():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    import lm_block_step
    return lm_block_step


def n(t):
    return t.double().cpu().numpy()


def oracle_gradients(pb):
    """(losses, G, dx) of the chain in 64 bits."""
    p = {k: n(v) for k, v in pb.slices(pb.w).items()}
    x, N = n(pb.x), pb.N
    y, mean, rstd = L.layer_norm(x, p["gamma"], p["beta"], 1e-5)
    a, z = L.linear(y, p["W1"], p["b1"], "gelu")
    h, _ = L.linear(a, p["W2"], p["b2"], residual=x)
    losses, _, dh, GV = L.softmax_xent(h, p["V"], pb.y.cpu().numpy(), N)
    da, G2, Gb2 = L.linear_grad(dh, None, a, p["W2"], "none", N)
    dn, G1, Gb1 = L.linear_grad(da, z, y, p["W1"], "gelu", N)
    dx, Gn = L.layer_norm_grad(dn, x, mean, rstd, p["gamma"], N)
    return losses, np.concatenate([Gn, G1, Gb1, G2, Gb2, GV.reshape(N, -1)], 1), dx + dh


@pytest.mark.parametrize("sizes", [dict(N=3, n_c=20, C=48, F=72, V=70), dict(N=4, n_c=130, C=264, F=520, V=300)])
def test_gradients_match_the_oracle(ex, sizes):
    """fp32 activations.  Tolerances: every operator of the chain of six is good to 2^-17 (the products' operands, sums,
    activations) of the largest element, and one takes the errors of those before it by its matrix, whose rows have norms of
    about 1, or by rstd, about 1: not more than tenfold over the chain, 10 * 6 * 2^-17 = 5e-4 of the largest element."""
    pb = ex.Problem(dtype=torch.float32, **sizes)
    loss, G, dx = ex.gradients(pb)
    losses, want, want_dx = oracle_gradients(pb)
    assert abs(loss.item() - losses.mean()) <= 1e-5 * losses.mean()
    for k, at in pb.at.items():
        assert rel_inf(n(G[:, at]), want[:, at]) <= 5e-4, k
    assert rel_inf(n(dx), want_dx) <= 5e-4


def test_a_worker_alone_computes_the_same_gradient(ex):
    """Rows of bf16: a chunk alone may sum dX of the head and of W2 in other ranges, which moves roundings of bf16 by one step,
    2^-8; they enter the gradients through sums over 40 points that such steps of both signs leave at no more than 2^-7 of
    the largest element."""
    pb = ex.Problem(N=6, n_c=40, C=136, F=200, V=300)
    G = ex.gradients(pb)[1]
    for chunk in (0, 5):
        got = ex.worker_gradient(pb, chunk)
        for k, at in pb.at.items():
            assert rel_inf(n(got[at]), n(G[chunk, at])) <= 2 ** -7, k


def test_a_step_with_the_code(ex):
    """All chunks finished: the decoded gradient is the sum of the chunk gradients, matrices move by the oracle's orthogonalised
    momentum of it and everything else by its mean."""
    pb = ex.Problem(N=6, n_c=32, C=64, F=136, V=100, dtype=torch.float32)
    w = pb.w.clone()
    for m in pb.momentum.values():
        m.uniform_(-1e-3, 1e-3)
    momentum = {k: n(m) for k, m in pb.momentum.items()}
    G = ex.gradients(pb)[1]
    psi = torch.full((1, 6), 3, dtype=torch.int32, device="cuda")
    g = ex.decoded(pb, G, psi)
    ref = O.run_pattern(n(pb.R), pb.order.cpu().numpy(), psi[0].cpu().numpy(), 6, n(G)).ghat
    assert rel_inf(n(g), ref) <= 1e-4
    assert rel_inf(n(g), n(G).sum(0)) <= 1e-4
    ex.update(pb, g, 0.5, 0.02)
    for k, at in pb.at.items():
        if k in momentum:
            shape = pb.shapes[k]
            W, M = L.muon_step(n(w[at]).reshape(shape), momentum[k], n(g[at]).reshape(shape), 0.02, 192,
                               scale=0.2 * max(shape) ** 0.5)
            # the update's values are below 1.2 (singular values) * lr * scale = 0.056, 4e-5 of them off in the 2-norm
            assert np.abs(n(pb.w[at]).reshape(shape) - W).max() <= 4e-5 * 0.056 * min(shape) ** 0.5 + 2 ** -24 * np.abs(W).max()
            assert rel_inf(n(pb.momentum[k]), M) <= 1e-6
        else:
            assert rel_inf(n(pb.w[at]), n(w[at]) - 0.5 / 192 * n(g[at])) <= 1e-6
    import paper_2405_19509_gb300 as gc
    gc.gc_status(pb.ws)


def test_a_captured_step_replays(ex):
    """Forward, backward, code and update in one graph with one workspace: the same bits as the calls."""
    def problem():
        return ex.Problem(N=4, n_c=40, C=72, F=328, V=129)

    def step(pb, G, psi):
        ex.update(pb, ex.decoded(pb, ex.gradients(pb, G=G)[1], psi), 0.5, 0.02)
    psi = torch.tensor([[3, 2, 3, 1]], dtype=torch.int32, device="cuda")
    a, b = problem(), problem()
    G = torch.empty(4, a.d, device="cuda")
    for _ in range(3):
        step(a, G, psi)
    torch.cuda.synchronize()
    start, momentum = b.w.clone(), {k: m.clone() for k, m in b.momentum.items()}
    step(b, G, psi)                                                    # the workspace reaches its size
    b.w.copy_(start)
    for k, m in momentum.items():
        b.momentum[k].copy_(m)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(b, G, psi)
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(a.w, b.w)
    for k in a.momentum:
        assert torch.equal(a.momentum[k], b.momentum[k])


def test_training_runs(ex):
    losses = ex.train(ex.Problem(N=6, n_c=64, C=128, F=256, V=500), 5)
    assert np.isfinite(losses).all()
