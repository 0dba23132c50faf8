"""gc_orthogonalize and gc_muon_step against 64-bit references.

Tolerances are in the 2-norm of a matrix O of singular values near 1, sqrt(m) of them.  The steps' slope is at most
3.4445^5 = 485 (singular values below 0.002 of the norm), which an error e of X0 is taken by.
fp32: X0 and every product are off by 2^-22 (two fp16 parts) and by 48 additions in a row, cut off by 2^-24 of a running sum of
two thirds on average, 1.9e-6.  An error of P is relative to its part of the singular values there; over the steps the slopes
on the way to the end multiply to 485 at most, and the errors of values that small are that much smaller than the rest: what
remains is the sum of five steps' three products, 15 * (1.9e-6 + 3 * 2^-22) = 4e-5.
bf16: O's own rounding, 2^-9 to 2^-8 and 1.7e-3 on average; X in A, P and the products' other operands off by 2^-12
(fp16 in one part): 2^-12 sqrt(1 / 3) on average, for three operands a step and five steps 15 * 1.4e-4 = 2.1e-3, taken by a
slope of up to 3.4 in the last: 7e-3 with the rounding."""
import numpy as np
import pytest
import torch

from oracle import lm_oracle as L

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
TOL = {torch.float32: 4e-5, torch.bfloat16: 7e-3}
COEFFS = (3.4445, -4.7750, 2.0315)


@pytest.fixture(scope="module")
def gc():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2405_19509_gb300 as m
    return m


def _randn(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")


def _gradient(seed, b, r, n):
    k = max(1, min(r, n) // 16)
    return _randn(seed, b, r, k) @ _randn(seed + 1, b, k, n) / k ** 0.5 + 0.5 * _randn(seed + 2, b, r, n)


def _ref(u, coeffs=COEFFS, steps=5, eps=1e-7):
    a, b, c = coeffs
    X = u.double()
    X = X / torch.linalg.matrix_norm(X)[:, None, None].clamp_min(eps)
    tall = X.shape[1] > X.shape[2]
    X = X.transpose(1, 2) if tall else X
    for _ in range(steps):
        A = X @ X.transpose(1, 2)
        X = a * X + (b * A + c * A @ A) @ X
    return X.transpose(1, 2) if tall else X


def _off(got, ref):
    return (torch.linalg.matrix_norm(got.double() - ref) / torch.linalg.matrix_norm(ref)).max().item()


def _lay(t, layout):
    """The same values: "strided" with rows apart on 16-byte boundaries, "ragged" on none, "beside" with the matrices of the
    batch side by side; NaN between."""
    b, r, n = t.shape
    if layout == "dense":
        return t.clone()
    if layout == "beside":
        big = torch.full((r, b, n + 3), float("nan"), dtype=t.dtype, device="cuda")
        big[:, :, :n] = t.transpose(0, 1)
        return big[:, :, :n].transpose(0, 1)
    pad, first = (16, 8) if layout == "strided" else (5, 3)
    width = -(-n // 8) * 8 + pad if layout == "strided" else n + pad
    big = torch.full((b, r + 1, width), float("nan"), dtype=t.dtype, device="cuda")
    big[:, :r, first:first + n] = t
    return big[:, :r, first:first + n]


SHAPES = [(1, 1, 1), (1, 1, 300), (2, 300, 1), (3, 5, 7), (1, 16, 2000), (1, 64, 257), (2, 257, 64), (1, 127, 130), (1, 128, 128),
          (2, 129, 500), (1, 500, 129), (12, 200, 200), (1, 256, 257), (3, 257, 255), (1, 300, 1111), (1, 1111, 300), (1, 520, 520),
          (5, 600, 700), (1, 1000, 1031)]


@pytest.mark.parametrize("x", ["f32", "bf16"])
@pytest.mark.parametrize("layout", ["dense", "strided", "ragged", "beside"])
@pytest.mark.parametrize("b,r,n", SHAPES)
def test_orthogonalize(gc, b, r, n, layout, x):
    u = _lay(_gradient(b + r + n, b, r, n).to(TYPES[x]), layout)
    out = _lay(torch.full((b, r, n), -77.0, dtype=u.dtype, device="cuda"), layout)
    ws = gc.Workspace()
    got = gc.gc_orthogonalize(u, out=out, ws=ws)
    gc.gc_status(ws)
    assert got is out and _off(got, _ref(u)) <= TOL[u.dtype]
    if layout in ("strided", "ragged"):
        assert torch.isnan(out._base).sum() == out._base.numel() - b * r * n       # nothing between the rows is written
    if b == 1:
        assert torch.equal(gc.gc_orthogonalize(u[0], ws=ws), got[0])
    again = gc.gc_orthogonalize(u, out=u, ws=ws)
    assert torch.equal(again, got)


@pytest.mark.parametrize("b,r,n", [(1, 2048, 2200), (2, 1024, 4096), (1, 4096, 1024), (1, 8, 100000), (40, 130, 100), (300, 17, 33),
                                   (1, 2100, 65)])
@pytest.mark.parametrize("x", ["f32", "bf16"])
def test_large(gc, b, r, n, x):
    u = _gradient(r + n, b, r, n).to(TYPES[x])
    assert _off(gc.gc_orthogonalize(u), _ref(u)) <= TOL[u.dtype]


@pytest.mark.parametrize("b,r,n", [(3, 78, 78), (1, 200, 200), (1, 184, 1344), (1, 1000, 181), (2, 256, 256), (3, 886, 1304)])
def test_five_steps_in_fp32_end_within_1e_5(gc, b, r, n):
    """What additions cut off is given back on average, so the module's 1.9e-6 a product is left with its spread: the cut
    is between 3/4 and 3/2 of its mean, by the significand, a fifth of 1.2e-6 in the 2-norm; with two operands and a result
    rounded by 2^-22 (sqrt(1 / 3) of it in the 2-norm) sqrt(0.24^2 + 3 * 0.14^2) = 0.34e-6 a product, independent from
    product to product: 0.34e-6 sqrt(15) = 1.3e-6, taken by slopes of up to 3.4 in each of the last two steps: below 1e-5, with
    a term for X0, 0.14e-6 times 485 beside the share, below a hundredth, of the singular values that are so small."""
    u = _gradient(b + r + n, b, r, n)
    assert _off(gc.gc_orthogonalize(u), _ref(u)) <= 1e-5


def test_reference_is_the_oracle():
    u = _gradient(1, 2, 9, 5)
    assert np.allclose(_ref(u)[1].cpu(), L.orthogonalize(u[1].double().cpu().numpy()))


@pytest.mark.parametrize("coeffs,steps", [((1.5, -0.5, 0.0), 1), ((1.875, -1.25, 0.375), 3), ((2.0, -1.5, 0.5), 8), (COEFFS, 1), (COEFFS, 2)])
@pytest.mark.parametrize("b,r,n", [(1, 100, 300), (2, 70, 40)])
def test_other_coefficients_and_steps(gc, b, r, n, coeffs, steps):
    u = _gradient(r, b, r, n)
    assert _off(gc.gc_orthogonalize(u, coeffs=coeffs, steps=steps), _ref(u, coeffs, steps)) <= TOL[u.dtype] * max(1, steps / 5)


@pytest.mark.parametrize("scale", [1e-38, 1e-30, 1e-12, 1e12, 1e25, 3e37])
def test_any_size_of_values(gc, scale):
    """The norm's squares leave fp32's range; the result is that of values near 1, but for the rounding of small ones (a
    value of 1e-38 keeps 2^-23 of itself)."""
    u = _gradient(3, 1, 60, 90).clamp(-8, 8) * scale
    assert _off(gc.gc_orthogonalize(u, eps=0.0), _ref(u, eps=0.0)) <= 4e-5


@pytest.mark.parametrize("kind", ["decay", "rank", "one"])
def test_spectra(gc, kind):
    """Singular values over four decades, a low rank, a single entry.  Of rank 3 the other 93 singular values are what rounding
    leaves, and the steps enlarge it: 2^-22 of X0 by 3.4445^5 = 485, and the 1.9e-6 + 3 * 2^-22 = 2.6e-6 of each of the next
    values of X by what steps are left, 141 + 41 + 12 + 3.4; together 1.16e-4 + 5.1e-4, beside |O| >= 0.7 sqrt(3): 5.2e-4."""
    tol = 5.2e-4 if kind == "rank" else 4e-5
    r, n = 96, 200
    if kind == "decay":
        u = torch.linalg.qr(_randn(1, r, r))[0] @ torch.diag(torch.logspace(0, -4, r, device="cuda")) @ torch.linalg.qr(_randn(2, n, n))[0][:r]
    elif kind == "rank":
        u = _randn(3, r, 3) @ _randn(4, 3, n)
    else:
        u = torch.zeros(r, n, device="cuda")
        u[5, 7] = -3.0
    u = u[None]
    assert _off(gc.gc_orthogonalize(u), _ref(u)) <= tol
    assert _off(gc.gc_orthogonalize(u.transpose(1, 2).contiguous()), _ref(u).transpose(1, 2)) <= tol


def test_zeros_and_values_that_are_not_finite(gc):
    u = _gradient(7, 4, 40, 70)
    want = gc.gc_orthogonalize(u)
    u[0] = 0
    u[1, 3, 4] = float("inf")
    u[2, 5, 6] = float("nan")
    got = gc.gc_orthogonalize(u)
    assert not got[0].any() and torch.isnan(got[1]).all() and torch.isnan(got[2]).all() and torch.equal(got[3], want[3])
    assert torch.isnan(gc.gc_orthogonalize(u[:1], eps=0.0)).all()
    tiny = torch.full((1, 2, 3), 1e-9, device="cuda")
    assert _off(gc.gc_orthogonalize(tiny, eps=1.0), _ref(tiny, eps=1.0)) <= TOL[u.dtype]


def _step(gc, w, m, g, **kw):
    gc.gc_muon_step(w, m, g, 0.02, 777, **kw)


@pytest.mark.parametrize("nesterov", [True, False])
@pytest.mark.parametrize("layout", ["dense", "strided", "ragged", "beside"])
@pytest.mark.parametrize("b,r,n", [(1, 1, 1), (3, 5, 7), (1, 257, 64), (12, 200, 200), (1, 1031, 300), (1, 300, 1111), (2, 512, 640)])
def test_muon(gc, b, r, n, layout, nesterov):
    """w beside its own rounding: the update, in the 2-norm, to the tolerance of O and 2^-23 of w."""
    w, m, g = _lay(_randn(1, b, r, n), layout), _lay(_gradient(5, b, r, n) * 0.1, layout), _lay(_gradient(9, b, r, n) * 30, layout)
    G, M, W = (t.double() for t in (g, m, w))
    M = 0.9 * M + G / 777
    O = _ref(G / 777 + 0.9 * M if nesterov else M)
    W = (1 - 0.02 * 0.1) * W - 0.02 * 3.0 * O
    ws = gc.Workspace()
    keep = g.clone()
    _step(gc, w, m, g, mu=0.9, nesterov=nesterov, weight_decay=0.1, scale=3.0, ws=ws)
    gc.gc_status(ws)
    assert torch.equal(g, keep)
    assert ((m.double() - M).abs() <= 2.0 ** -22 * (M.abs() + G.abs() / 777)).all()
    tol = 0.06 * TOL[torch.float32] * torch.linalg.matrix_norm(O) + 2.0 ** -23 * torch.linalg.matrix_norm(W)
    assert (torch.linalg.matrix_norm(w.double() - W) <= tol).all()
    if layout in ("strided", "ragged"):
        assert torch.isnan(w._base).sum() == w._base.numel() - b * r * n == torch.isnan(m._base).sum()


def test_muon_is_the_oracle(gc):
    w, m, g = _randn(1, 20, 30), _randn(2, 20, 30), _randn(3, 20, 30)
    n = lambda t: t.double().cpu().numpy()
    W, M = L.muon_step(n(w), n(m), n(g), 0.1, 5, weight_decay=0.01, scale=0.5)
    gc.gc_muon_step(w, m, g, 0.1, 5, weight_decay=0.01, scale=0.5)
    assert np.allclose(n(w), W, atol=1e-5) and np.allclose(n(m), M, atol=1e-6)


def test_slices_of_a_parameter_vector(gc):
    """w and g as a user has them: slices of the parameters and of the decoded gradient, which keep the rest."""
    C, F = 70, 90
    w, m, g = _randn(1, 11 + F * C + 5), torch.zeros(F, C, device="cuda"), _randn(2, 11 + F * C + 5)
    s = slice(11, 11 + F * C)
    want = w[s].view(F, C).clone()
    gc.gc_muon_step(want, m.clone(), g[s].view(F, C).clone(), 0.1, 9)
    before = w.clone()
    gc.gc_muon_step(w[s].view(F, C), m, g[s].view(F, C), 0.1, 9)
    assert torch.equal(w[s].view(F, C), want) and torch.equal(w[:11], before[:11]) and torch.equal(w[11 + F * C:], before[11 + F * C:])


def test_a_matrix_alone_and_in_a_batch(gc):
    """The same update to rounding, whatever the batch (the sums' ranges may differ)."""
    u = _gradient(11, 9, 100, 260)
    got = gc.gc_orthogonalize(u)
    for i in (0, 8):
        assert _off(got[i:i + 1], gc.gc_orthogonalize(u[i:i + 1]).double()) <= 2 * TOL[u.dtype]


def test_an_empty_batch(gc):
    assert gc.gc_orthogonalize(torch.empty(0, 3, 4, device="cuda")).shape == (0, 3, 4)


def test_on_another_stream_and_in_a_graph(gc):
    w, m, g = _randn(1, 2, 300, 520), _randn(2, 2, 300, 520), _randn(3, 2, 300, 520)
    W, M = w.clone(), m.clone()
    for _ in range(3):
        _step(gc, W, M, g)
    torch.cuda.synchronize()
    ws = gc.Workspace()
    s = torch.cuda.Stream()
    w2, m2 = w.clone(), m.clone()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        for _ in range(3):
            _step(gc, w2, m2, g, ws=ws)
    s.synchronize()
    assert torch.equal(w2, W) and torch.equal(m2, M)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _step(gc, w, m, g, ws=ws)
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(w, W) and torch.equal(m, M)
    gc.gc_status(ws)


def test_stall_times_out_then_recovers(gc):
    u = _gradient(5, 1, 300, 400)
    want = gc.gc_orthogonalize(u)
    ws = gc.Workspace()
    gc.gc_set_wait_limit(1 << 22)
    try:
        gc.gc_inject_stall(gc.GC_STALL_MUON)
        gc.gc_orthogonalize(u, ws=ws)
        torch.cuda.synchronize()
        with pytest.raises(gc.GCError) as e:
            gc.gc_status(ws)
        assert e.value.code == -5
    finally:
        gc.gc_inject_stall(0)
        gc.gc_set_wait_limit(0)
    got = gc.gc_orthogonalize(u, ws=ws)
    gc.gc_status(ws)
    assert torch.equal(got, want)
