"""gc_orthogonalize and gc_muon_step where tiles on the tensor cores take the work (both sides above 64, which every test
asserts): digits of results by the kind of matrix, small norms, values that are not finite."""
import pytest
import torch

from test_gpu_muon import TYPES, _gradient, _off, _randn, _ref, gc  # noqa: F401

pytestmark = pytest.mark.gpu


def _by_tiles(gc, u):
    b, r, n = u.shape
    assert gc.lib.gc_orthogonalize_workspace(b, r, n, 1 if u.dtype == torch.bfloat16 else 0) > 256
    return u


def _sparse(kind):
    """Matrices whose products have few terms: adding zeros cuts nothing off."""
    if kind == "identity":
        return torch.eye(512, device="cuda")[None]
    if kind == "odd identity":
        return torch.eye(519, device="cuda")[None]
    if kind == "identities":
        return torch.eye(512, device="cuda").repeat(12, 1, 1)
    if kind == "permuted":
        return (torch.eye(700, 1000, device="cuda")[torch.randperm(700, generator=torch.Generator().manual_seed(1)).cuda()])[None]
    if kind == "diagonal":
        return torch.diag(0.5 + torch.rand(520, generator=torch.Generator(device="cuda").manual_seed(2), device="cuda"))[None]
    if kind == "four equal":
        u = torch.zeros(1, 520, 600, device="cuda")
        for i in range(4):
            u[0, 100 * i + 7, 130 * i + 3] = -2.0
        return u
    if kind == "four equal, many":
        return _sparse("four equal").repeat(12, 1, 1)
    if kind == "blocks":
        return torch.block_diag(*_randn(3, 16, 32, 40))[None]
    if kind == "few rows":                             # an output matrix of which few words were seen
        u = torch.zeros(1, 1000, 520, device="cuda")
        u[0, ::29] = _randn(4, 35, 520)
        return u
    u = torch.zeros(1, 520, 1031, device="cuda")       # few columns: units that were never active
    u[0, :, ::17] = _randn(5, 520, 61)
    return u


SPARSE = ["identity", "odd identity", "identities", "permuted", "diagonal", "four equal", "four equal, many", "blocks", "few rows"]


@pytest.mark.parametrize("kind", SPARSE)
@pytest.mark.parametrize("tall", [False, True])
def test_sums_of_few_terms_keep_their_digits(gc, kind, tall):
    """What an addition in tensor memory cuts off depends on what is there: sums of few terms lose nothing or little.  gc.h states
    1e-5 for all matrices of full rank, and for those whose other singular values are exactly 0."""
    u = _by_tiles(gc, _sparse(kind))
    ref = _ref(u)
    if tall:
        u, ref = u.transpose(1, 2).contiguous(), ref.transpose(1, 2)
    assert _off(gc.gc_orthogonalize(u), ref) <= 1e-5


@pytest.mark.parametrize("b,r,n", [(3, 78, 78), (1, 200, 200), (1, 184, 1344), (1, 1000, 181), (2, 256, 256), (3, 886, 1304), (1, 1024, 1024),
                                   (1, 130, 4100)])
def test_dense_matrices_keep_their_digits(gc, b, r, n):
    """A cut is half of 2^-24 on average, 0.32e-6 a product of 16 additions, and 0.96e-6 a step; singular values between 0.7 and 1.2
    are taken by slopes of up to 1.7 in every step after it, 1 + 1.7 + .. + 1.7^4 = 18.9 of them: 1.8e-5 if all were of one
    sign.  gc.h states 1e-5."""
    u = _by_tiles(gc, _gradient(b + r + n, b, r, n))
    assert _off(gc.gc_orthogonalize(u), _ref(u)) <= 1e-5


@pytest.mark.parametrize("b,r,n", [(1, 200, 200), (1, 184, 1344), (2, 300, 256), (1, 1024, 4096), (1, 2048, 520)])
def test_bf16_matrices_are_rounded_once(gc, b, r, n):
    """The steps of a bf16 matrix keep an fp32 one's digits: a value v off by e before it is rounded ends at most 2 e further from v
    than v's own rounding.  e: 3 K / 16 additions in each of 15 products, cut off by half of 2^-24 on average of a running sum of
    two thirds, and 3 * 0.14e-6 for 22 bits of operands and results."""
    u = _by_tiles(gc, _gradient(b + r + n, b, r, n).to(torch.bfloat16))
    ref = _ref(u)
    K = (max(r, n) + 2 * min(r, n)) / 3
    e = 15 * (3 * K / 16 * 2.0 ** -25 * 2 / 3 + 0.42e-6)
    assert _off(gc.gc_orthogonalize(u), ref) <= _off(ref.to(torch.bfloat16), ref) + 2 * e


COEFFS = [((3.4445, -4.7750, 2.0315), 5), ((1.875, -1.25, 0.375), 20), ((1.5, -0.5, 0.0), 64), ((0.5, 0.0, 0.0), 40)]


@pytest.mark.parametrize("coeffs,steps", COEFFS)
@pytest.mark.parametrize("below", [1.0, 1e-1, 1e-3, 1e-5, 1.5e-6, 1e-9, 1e-20])
@pytest.mark.parametrize("r,n", [(300, 400), (1000, 1000)])
def test_norms_below_eps(gc, r, n, below, coeffs, steps):
    """u far below eps starts the steps far below 1, and may reach 1 in many; it keeps the digits of any other.  Beyond five steps the
    polynomials' slope near 1 is below 1, so that errors do not add up."""
    u = _gradient(r, 1, r, n)
    u = _by_tiles(gc, u / torch.linalg.matrix_norm(u)[:, None, None])
    u, eps = u * 2.0 ** -10, 2.0 ** -10 / below
    ref = _ref(u, coeffs, steps, eps)
    assert _off(gc.gc_orthogonalize(u, coeffs=coeffs, steps=steps, eps=eps), ref) <= 1e-5


def test_norms_of_a_batch_are_its_matrices(gc):
    """Matrices of a batch with norms above, below and far below eps, and zeros."""
    u = _by_tiles(gc, _gradient(3, 5, 130, 200))
    u = u / torch.linalg.matrix_norm(u)[:, None, None] * torch.tensor([3.0, 0.5, 1e-4, 1e-12, 0.0], device="cuda")[:, None, None]
    got, ref = gc.gc_orthogonalize(u, eps=1.0), _ref(u, eps=1.0)
    for i in range(4):
        assert _off(got[i:i + 1], ref[i:i + 1]) <= 1e-5
    assert not got[4].any()
    w, m = torch.zeros_like(u), torch.zeros_like(u)
    gc.gc_muon_step(w, m, u, 1.0, 1, mu=0.5, nesterov=False, eps=1.0)
    for i in range(4):
        assert _off(-w[i:i + 1], ref[i:i + 1]) <= 1e-5


@pytest.mark.parametrize("x", ["f32", "bf16"])
def test_zeros_and_values_that_are_not_finite(gc, x):
    """A matrix of zeros stays one, one with an infinity or NaN becomes NaN, and no other matrix of the batch changes."""
    u = _by_tiles(gc, _gradient(7, 5, 130, 200).to(TYPES[x]))
    want = gc.gc_orthogonalize(u)
    u[0] = 0
    u[1, 3, 4] = float("inf")
    u[2, 129, 199] = float("nan")
    u[3, 0, 0] = float("-inf")
    got = gc.gc_orthogonalize(u)
    assert not got[0].any() and all(torch.isnan(got[i]).all() for i in (1, 2, 3)) and torch.equal(got[4], want[4])
    assert torch.isnan(gc.gc_orthogonalize(u[:1], eps=0.0)).all()


def test_a_step_of_values_that_are_not_finite(gc):
    w, m, g = (_by_tiles(gc, _randn(s, 3, 130, 200)) for s in (1, 2, 3))
    W, M = w.clone(), m.clone()
    gc.gc_muon_step(W, M, g, 0.02, 9)
    g[1, 5, 6] = float("inf")
    gc.gc_muon_step(w, m, g, 0.02, 9)
    assert torch.isnan(w[1]).all() and all(torch.equal(w[i], W[i]) and torch.equal(m[i], M[i]) for i in (0, 2))


@pytest.mark.parametrize("r,n", [(130, 200), (1000, 300)])
@pytest.mark.parametrize("scale", [1e-38, 1e-30, 1e-12, 1e12, 1e25, 3e37])
def test_any_size_of_values(gc, r, n, scale):
    """The norm's squares leave fp32's range.  The result is that of the values as they are stored: 1e-5 as for values near 1."""
    u = _by_tiles(gc, _gradient(3, 1, r, n).clamp(-8, 8) * scale)
    assert _off(gc.gc_orthogonalize(u, eps=0.0), _ref(u, eps=0.0)) <= 1e-5


@pytest.mark.parametrize("r,n", [(96, 200), (520, 520), (1000, 300)])
def test_low_rank(gc, r, n):
    """Of rank 3 the other singular values are what rounding leaves of them, and the steps enlarge it by up to 3.4445^5 = 485: a
    spread of 2^-22 sqrt(1 / 3) of X0's values, 1.4e-7, and 3 * 2^-22 sqrt(1 / 3) of each of the next X, by what steps are
    left, 485, 141, 41, 12 and 3.4: 6.8e-5 + 8.3e-5, beside |O| of about |X| then."""
    u = _by_tiles(gc, (_randn(3, r, 3) @ _randn(4, 3, n))[None])
    assert _off(gc.gc_orthogonalize(u), _ref(u)) <= 1.6e-4


@pytest.mark.parametrize("x,off", [("bf16", 2e-5), ("f32", 1e-5)])
@pytest.mark.parametrize("r,n", [(80, 40000), (2048, 2100)])
def test_long_sums_are_not_cut_off(gc, r, n, x, off):
    """Rounding leaves the size of the result what it is on average.  Four K blocks (two in fp32) of three products are cut off by
    up to 40 (16) times 2^-24 of a running sum of a half, 1.2e-6 (0.5e-6) a product; fifteen products 1.8e-5 (0.75e-5)."""
    u = _by_tiles(gc, _gradient(r, 1, r, n).to(TYPES[x]))
    ref = _ref(u)
    assert abs(((gc.gc_orthogonalize(u).double() * ref).sum() / (ref * ref).sum()).item() - 1) <= off
