"""The operators of a language model's output end together, as examples/lm_head_step.py runs them."""
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
    import lm_head_step
    return lm_head_step


def test_a_worker_alone_computes_the_same_bits(ex):
    """The mask is that of the points, and at these sizes the sums run in one order."""
    pb = ex.Problem(N=6, n_c=40, C=136, V=300)
    G = ex.gradients(pb, 3)[1]
    for chunk in (0, 2, 5):
        assert torch.equal(ex.worker_gradient(pb, 3, chunk), G[chunk])
    assert not torch.equal(ex.worker_gradient(pb, 4, 2), G[2])     # another iteration, another mask


def test_gradients_match_the_oracle(ex):
    """fp32 activations: the chain of forward and backward in 64 bits.  Tolerances: every factor of the
    chain is good to 2^-15 (the products' operands) of values that the chain does not amplify by more than
    ten: 1e-3 of the largest element."""
    pb = ex.Problem(N=3, n_c=20, C=48, V=70, dtype=torch.float32)
    loss, G, dx, dres = ex.gradients(pb, 1)
    n = lambda t: t.double().cpu().numpy()
    gamma, beta, W = (n(t) for t in pb.slices(pb.w))
    h = L.dropout(n(pb.branch), pb.p, pb.seed, 1, 0, n(pb.residual))
    y, mean, rstd = L.layer_norm(h, gamma, beta, 1e-5)
    losses, _, dX, GW = L.softmax_xent(y, W, pb.y.cpu().numpy(), 3)
    dh, Gn = L.layer_norm_grad(dX, h, mean, rstd, gamma, 3)
    assert abs(loss.item() - losses.mean()) <= 1e-5 * losses.mean()
    assert rel_inf(n(dres), dh) <= 1e-3
    assert rel_inf(n(dx), L.dropout(dh, pb.p, pb.seed, 1)) <= 1e-3
    assert rel_inf(n(G[:, :96]), Gn) <= 1e-3
    assert rel_inf(n(G[:, 96:]), GW.reshape(3, -1)) <= 1e-3


def test_the_gradients_are_encoded_and_decoded(ex):
    """All chunks finished: the decoded gradient is the sum of the chunk gradients."""
    import paper_2405_19509_gb300 as gc
    pb = ex.Problem(N=6, n_c=32, C=64, V=257)
    G = ex.gradients(pb, 0)[1]
    psi = torch.full((1, 6), 3, dtype=torch.int32, device="cuda")
    T = gc.gc_encode(pb.R, pb.ell, pb.order, 6, 6, 3, psi, G, ws=pb.ws)
    got = gc.gc_decode_tx(pb.R, pb.ell, 6, T, pb.d)
    ref = O.run_pattern(pb.R.cpu().numpy(), pb.order.cpu().numpy(), psi[0].cpu().numpy(), 6,
                        G.double().cpu().numpy()).ghat
    assert rel_inf(got[0].cpu().numpy(), ref) <= 1e-4
    assert rel_inf(got[0].cpu().numpy(), G.double().sum(0).cpu().numpy()) <= 1e-4


def test_training_lowers_the_loss(ex):
    losses = ex.train(ex.Problem(N=6, n_c=64, C=128, V=500), 30)
    assert np.isfinite(losses).all() and np.mean(losses[-3:]) < 0.7 * losses[0]
