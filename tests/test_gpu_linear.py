"""gc_linear and gc_linear_backward against 64-bit references.

Tolerances, element by element, with S the sum of the products' magnitudes.  Operands: bf16 enters as it is; an fp32 value
beside bf16 as hi + lo, off by 2^-17; fp32 beside fp32 as three parts, each off by 2^-26, without the products that are
below 2^-24: 2^-23 S.  A sum of K products in tensor memory: K / 16 additions for each of its 1, 2, 3 or 6 products of
parts, and 32 more to join ranges, each off by at most 2^-23 S.  Activations: 2^-20 (1 + |z|), slopes 2^-19; no
slope of an activation is past 1.13.  bf16 results are rounded by 2^-8 of themselves, fp32 ones by 2^-24."""
import numpy as np
import pytest
import torch

from oracle import lm_oracle as L

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
PAIRS = [("bf16", "bf16"), ("f32", "f32"), ("bf16", "f32"), ("f32", "bf16")]
ACTS = ["none", "relu", "gelu", "gelu_tanh", "silu"]
R = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


@pytest.fixture(scope="module")
def gc():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2405_19509_gb300 as m
    return m


def _code(gc, act):
    return {"none": gc.GC_ACT_NONE, "relu": gc.GC_ACT_RELU, "gelu": gc.GC_ACT_GELU, "gelu_tanh": gc.GC_ACT_GELU_TANH,
            "silu": gc.GC_ACT_SILU}[act]


class Maker:
    """Matrices of one seed; "strided": rows apart on 16-byte boundaries, "ragged": on none, NaN between them."""

    def __init__(self, seed, layout="dense"):
        self.g = torch.Generator(device="cuda").manual_seed(seed)
        self.layout = layout

    def randn(self, *shape):
        return torch.randn(*shape, generator=self.g, device="cuda")

    def mat(self, rows, cols, dtype, scale=1.0):
        a = (scale * self.randn(rows, cols)).to(dtype)
        if self.layout == "dense":
            return a
        pad, first = (16, 8) if self.layout == "strided" else (5, 3)
        width = cols + pad if self.layout == "ragged" else -(-cols // 8) * 8 + pad
        big = torch.full((rows, width), float("nan"), dtype=dtype, device="cuda")
        big[:, first:first + cols] = a
        return big[:, first:first + cols]

    def out(self, rows, cols, dtype):
        """(an output, the buffer around it)"""
        pad, first = {"dense": (0, 0), "strided": (16, 8), "ragged": (5, 3)}[self.layout]
        width = -(-cols // 8) * 8 + pad if self.layout == "strided" else cols + pad
        big = torch.full((rows, width), -77.0, dtype=dtype, device="cuda")
        return big[:, first:first + cols], big


def _untouched(view, big):
    first = view.storage_offset()
    return bool((big[:, :first] == -77).all()) and bool((big[:, first + view.shape[1]:] == -77).all())


def _act(z, act):
    if act == "relu":
        return z.clamp_min(0)
    if act == "gelu":
        return z * torch.special.ndtr(z)
    if act == "gelu_tanh":
        return z * torch.special.expit(2 * (2 / np.pi) ** 0.5 * (z + 0.044715 * z ** 3))
    return z * torch.special.expit(z) if act == "silu" else z


def _slope(z, act):
    z = z.clone().requires_grad_()
    with torch.enable_grad():
        y = torch.relu(z) if act == "relu" else _act(z, act)
        return torch.autograd.grad(y.sum(), z)[0]


def _parts(a, b):
    return (0.0, 1) if a == b == torch.bfloat16 else (2.0 ** -17, 2) if a == torch.bfloat16 else (2.0 ** -23, 6)


def _ref_linear(x, W, bias, act, residual):
    off, prod = _parts(x.dtype, W.dtype)
    X, V = x.double(), W.double()
    z, S = X @ V.T, X.abs() @ V.abs().T
    tz = (off + (x.shape[1] / 16 * prod + 32) * 2.0 ** -23) * S
    if bias is not None:
        z = z + bias.double()
        tz = tz + 2.0 ** -23 * z.abs()
    y = _act(z, act)
    ty = 1.13 * tz + (0 if act in ("none", "relu") else 2.0 ** -20 * (1 + z.abs()))
    if residual is not None:
        y = y + residual.double()
        ty = ty + 2.0 ** -23 * y.abs()
    r = R[x.dtype]
    return {"y": (y, ty * (1 + r) + r * y.abs()), "z": (z, tz * (1 + r) + r * z.abs())}


def _ref_grad(dy, z, x, W, act, N):
    bf = x.dtype == torch.bfloat16
    off, prod = _parts(x.dtype, W.dtype)
    T, F = dy.shape
    d, td = dy.double(), torch.zeros_like(dy, dtype=torch.double)
    if act != "none":
        td = d.abs() * (2.0 ** -19 if act != "relu" else 0) + 2.0 ** -24 * d.abs()
        d = d * _slope(z.double(), act)
    V, X = W.double(), x.double()
    steps = lambda K, p: (K / 16 * p + 32) * 2.0 ** -23
    dx = d @ V
    tdx = (td + d.abs() * ((2.0 ** -8 if bf and act != "none" else 0) + off + steps(F, prod))) @ V.abs()
    tdx = tdx * (1 + R[x.dtype]) + R[x.dtype] * dx.abs()
    c = lambda a: a.view(N, T // N, -1)
    in_g = 2.0 ** -23 if not bf else 2.0 ** -17 if act != "none" else 0.0
    tg = td + d.abs() * (in_g + steps(T // N, 6 if not bf else 2))
    G = torch.bmm(c(d).transpose(1, 2), c(X)).flatten(1)
    tG = torch.bmm(c(tg).transpose(1, 2), c(X.abs())).flatten(1)
    tGb = (c(td) + c(d.abs()) * (T // N + 1) * 2.0 ** -24).sum(1)
    return {"dx": (dx, tdx), "G": (G, tG), "Gb": (c(d).sum(1), tGb)}


def _close(got, ref, what):
    value, tol = ref
    off = (got.double() - value).abs()
    assert bool((off <= tol + 1e-30).all()), f"{what}: {(off - tol).max().item():.3e} past its tolerance"


SHAPES = [(1, 1, 1), (1, 64, 257), (1, 2048, 5000), (2, 300, 33), (3, 7, 11), (5, 1000, 4003), (17, 8, 8), (64, 520, 96), (77, 1000, 2003),
          (128, 64, 256), (129, 4096, 40), (192, 64, 256), (300, 200, 1000), (700, 1031, 129), (2048, 136, 513)]


@pytest.mark.parametrize("x,w", PAIRS)
@pytest.mark.parametrize("layout", ["dense", "strided", "ragged"])
@pytest.mark.parametrize("T,C,F", SHAPES)
def test_forward(gc, T, C, F, x, w, layout):
    for i, act in enumerate(ACTS):
        m = Maker(T + C + F + i, layout)
        X, W = m.mat(T, C, TYPES[x]), m.mat(F, C, TYPES[w], C ** -0.5)
        bias = 0.3 * m.randn(F) if i != 1 else None
        res = m.mat(T, F, TYPES[x]) if i % 2 else None
        y, yb = m.out(T, F, TYPES[x])
        z, zb = m.out(T, F, TYPES[x])
        ws = gc.Workspace()
        got = gc.gc_linear(X, W, bias, _code(gc, act), residual=res, y=y, z=z if i < 3 else False, ws=ws)
        gc.gc_status(ws)
        ref = _ref_linear(X, W, bias, act, res)
        _close(got["y"], ref["y"], f"y, {act}")
        assert _untouched(y, yb) and _untouched(z, zb)
        if i < 3:
            _close(got["z"], ref["z"], f"z, {act}")


GRADS = [(1, 1, 1, 1), (1, 1, 64, 257), (6, 32, 64, 256), (3, 5, 7, 11), (2, 64, 128, 512), (1, 300, 200, 1000), (4, 77, 1000, 1031),
         (5, 1, 40, 300), (1, 257, 72, 255), (2, 130, 520, 2049), (20, 20, 96, 700), (1, 3, 2048, 4000), (3, 500, 24, 3000)]


@pytest.mark.parametrize("x,w", PAIRS)
@pytest.mark.parametrize("layout", ["dense", "strided", "ragged"])
@pytest.mark.parametrize("N,n_c,C,F", GRADS)
def test_backward(gc, N, n_c, C, F, x, w, layout):
    for i, act in enumerate(ACTS):
        m = Maker(N + n_c + C + F + i, layout)
        T, t = N * n_c, TYPES[x]
        X, W = m.mat(T, C, t), m.mat(F, C, TYPES[w], C ** -0.5)
        z, dy = (m.mat(T, F, t, 1.5) if act != "none" else None), m.mat(T, F, t)
        dx, db = m.out(T, C, t)
        G, Gw = m.out(N, F * C, torch.float32)
        Gb, Gbw = m.out(N, F, torch.float32)
        ws = gc.Workspace()
        got = gc.gc_linear_backward(dy, X, W, N, n_c, z=z, act=_code(gc, act), dx=dx, G=G, Gb=Gb, ws=ws)
        gc.gc_status(ws)
        for k, v in _ref_grad(dy, z, X, W, act, N).items():
            _close(got[k], v, f"{k}, {act}")
        assert _untouched(dx, db) and _untouched(G, Gw) and _untouched(Gb, Gbw)


def test_reference_is_the_oracle():
    m = Maker(1)
    x, W, b, res, dy = m.mat(12, 10, torch.float32), m.mat(7, 10, torch.float32), m.randn(7), m.randn(12, 7), m.randn(12, 7)
    n = lambda t: t.double().cpu().numpy()
    for act in ACTS:
        ref = _ref_linear(x, W, b, act, res)
        y, z = L.linear(n(x), n(W), n(b), act, n(res))
        assert np.allclose(n(ref["y"][0]), y) and np.allclose(n(ref["z"][0]), z)
        ref = _ref_grad(dy, ref["z"][0].float(), x, W, act, 3)
        for k, v in zip(("dx", "G", "Gb"), L.linear_grad(n(dy), z.astype(np.float32), n(x), n(W), act, 3)):
            assert np.allclose(n(ref[k][0]), v)


@pytest.mark.parametrize("x", ["bf16", "f32"])
def test_a_chunk_alone_gives_the_same_bits(gc, x):
    """A worker that holds one chunk sends what any other sends for it, whatever tiles its call has."""
    for N, n_c, C, F in ((4, 150, 200, 777), (24, 256, 256, 512), (8, 1024, 512, 1024), (40, 3, 64, 128)):
        m = Maker(N + F)
        X, W, z, dy = m.mat(N * n_c, C, TYPES[x]), m.mat(F, C, TYPES[x]), m.mat(N * n_c, F, TYPES[x]), m.mat(N * n_c, F, TYPES[x])
        full = gc.gc_linear_backward(dy, X, W, N, n_c, z=z, act=gc.GC_ACT_GELU)
        for i in (0, N - 1):
            r = slice(i * n_c, (i + 1) * n_c)
            one = gc.gc_linear_backward(dy[r], X[r], W, 1, n_c, z=z[r], act=gc.GC_ACT_GELU)
            alone = gc.gc_linear_backward(dy[r], X[r], W, 1, n_c, z=z[r], act=gc.GC_ACT_GELU, dx=False)
            for k in ("G", "Gb"):
                assert torch.equal(one[k][0], full[k][i]) and torch.equal(alone[k][0], full[k][i])


@pytest.mark.parametrize("x,w", PAIRS)
def test_outputs_alone_and_repeated(gc, x, w):
    m = Maker(3)
    N, n_c, C, F = 3, 90, 136, 520
    X, W = m.mat(N * n_c, C, TYPES[x]), m.mat(F, C, TYPES[w])
    z, dy = m.mat(N * n_c, F, TYPES[x]), m.mat(N * n_c, F, TYPES[x])
    ws = gc.Workspace()
    call = lambda **k: gc.gc_linear_backward(dy, X, W, N, n_c, z=z, act=gc.GC_ACT_SILU, ws=ws, **k)
    full = call()
    again = call()
    assert all(torch.equal(full[k], again[k]) for k in full)
    for k in full:
        only = call(**{j: j == k for j in full})
        assert torch.equal(only[k], full[k]) if k != "dx" else (only[k] - full[k]).abs().max() <= 2 ** -7 * full[k].abs().max()
        assert all(only[j] is None for j in full if j != k)
    a = gc.gc_linear(X, W, act=gc.GC_ACT_SILU, z=True, ws=ws)
    b = gc.gc_linear(X, W, act=gc.GC_ACT_SILU, ws=ws)
    assert b["z"] is None and torch.equal(a["y"], b["y"])


@pytest.mark.parametrize("n_c", [8000, 9000])
def test_bias_gradients_alone_have_the_same_bits(gc, n_c):
    """Partial sums of few points are joined beside the products, of many in a launch of their own, alone always."""
    m = Maker(n_c)
    x, W, dy, z = (m.mat(*s, torch.bfloat16) for s in ((2 * n_c, 72), (130, 72), (2 * n_c, 130), (2 * n_c, 130)))
    all_ = gc.gc_linear_backward(dy, x, W, 2, n_c, z=z, act=gc.GC_ACT_SILU)
    alone = gc.gc_linear_backward(dy, x, W, 2, n_c, z=z, act=gc.GC_ACT_SILU, dx=False, G=False)["Gb"]
    assert torch.equal(all_["Gb"], alone)
    _close(alone, _ref_grad(dy, z, x, W, "silu", 2)["Gb"], "Gb")


@pytest.mark.parametrize("T", [1, 5, 300])
@pytest.mark.parametrize("x", ["bf16", "f32"])
def test_y_over_the_residual(gc, x, T):
    m = Maker(4)
    X, W, res = m.mat(T, 72, TYPES[x]), m.mat(300, 72, TYPES[x]), m.mat(T, 300, TYPES[x])
    want = gc.gc_linear(X, W, act=gc.GC_ACT_GELU, residual=res)["y"]
    got = gc.gc_linear(X, W, act=gc.GC_ACT_GELU, residual=res, y=res)["y"]
    assert got is res and torch.equal(got, want)


def test_no_rows(gc):
    x, W = torch.empty(0, 8, device="cuda"), torch.ones(5, 8, device="cuda")
    assert gc.gc_linear(x, W)["y"].shape == (0, 5)


@pytest.mark.parametrize("x,w", PAIRS)
@pytest.mark.parametrize("T", [4, 300])
def test_a_row_reaches_its_own_alone(gc, x, w, T):
    """Infinities, NaN and the end of the range in one row: the other rows keep their bits."""
    m = Maker(5)
    N, C, F = 2, 100, 520
    t = TYPES[x]
    X, W, z, dy = m.mat(T, C, t), m.mat(F, C, TYPES[w]), m.mat(T, F, t), m.mat(T, F, t)
    want = gc.gc_linear(X, W, act=gc.GC_ACT_RELU, z=True)
    back = gc.gc_linear_backward(dy, X, W, N, T // N, z=z, act=gc.GC_ACT_GELU)
    for bad in (float("inf"), float("-inf"), float("nan")):
        X2, dy2 = X.clone(), dy.clone()
        X2[1, 3] = bad
        dy2[1, 7] = bad
        got = gc.gc_linear(X2, W, act=gc.GC_ACT_RELU, z=True)
        rest = torch.arange(T, device="cuda") != 1
        assert all(torch.equal(got[k][rest], want[k][rest]) for k in got)
        assert not torch.isfinite(got["z"][1]).any()
        got = gc.gc_linear_backward(dy2, X, W, N, T // N, z=z, act=gc.GC_ACT_GELU)
        assert torch.equal(got["dx"][rest], back["dx"][rest]) and not torch.isfinite(got["dx"][1]).any()
        assert torch.equal(got["G"][1], back["G"][1]) and torch.equal(got["Gb"][1], back["Gb"][1])
        assert not torch.isfinite(got["G"][0].view(F, C)[7]).any() and torch.isfinite(got["G"][0].view(F, C)[8:]).all()
        assert not torch.isfinite(got["Gb"][0, 7]) and torch.isfinite(got["Gb"][0, 8:]).all()


def test_values_at_the_end_of_the_range(gc):
    """fp32's largest values round past bf16's; one of them in a row of zeros is itself in y, to 2^-23."""
    X = torch.zeros(3, 40, device="cuda")
    X[0, 5], X[1, 6], X[2, 7] = 3.4028234e38, -3.4028234e38, 2.0 ** -120
    W = torch.zeros(50, 40, device="cuda")
    W[:, 5], W[:, 6], W[:, 7] = 1.0, 0.5, 1.0
    got = gc.gc_linear(X, W)["y"]
    want = torch.stack([X[0, 5].repeat(50), 0.5 * X[1, 6].repeat(50), X[2, 7].repeat(50)])
    assert ((got.double() - want.double()).abs() <= 2.0 ** -22 * want.double().abs()).all()


@pytest.mark.parametrize("act", ["gelu", "gelu_tanh", "silu", "relu"])
def test_far_arguments(gc, act):
    """z far from 0: act(z) is z or 0 and its slope 1 or 0, with no overflow on the way."""
    z = torch.tensor([[1e4, -1e4, 1e19, -1e19, 3e38, -3e38, 200.0, -200.0, 0.0, 40.0]], device="cuda").T.contiguous()
    one = torch.ones(1, 1, device="cuda")
    y = gc.gc_linear(z, one, act=_code(gc, act))["y"]
    assert torch.allclose(y, z.clamp_min(0), rtol=2e-6, atol=0)
    d = gc.gc_linear_backward(torch.ones_like(z), z, one, 1, 10, z=z, act=_code(gc, act), G=False, Gb=False)["dx"]
    want = (z > 0).float()
    if act != "relu":
        want[8] = 0.5
    assert torch.allclose(d, want, rtol=0, atol=1e-6)


@pytest.mark.parametrize("act", ["gelu", "gelu_tanh", "silu"])
def test_gradients_against_differences(gc, act):
    """Central differences of the GPU's own y along a direction, of fp32 values of order 1: each of 600 values is off by some
    2^-20, over 2 t with t = 2^-7: 600^0.5 2^-14 = 1.5e-3; the cubic term t^2 / 6 f''' times the directions' size, 600 times
    10^-5 5^1.5 at most: 7e-2; the derivative is of order 100."""
    m = Maker(11)
    N, n_c, C, F = 2, 10, 25, 30
    X, W, b, dy = m.mat(N * n_c, C, torch.float32), m.mat(F, C, torch.float32, 0.2), m.randn(F), m.randn(N * n_c, F)
    s, q, r = m.randn(N * n_c, C), 0.2 * m.randn(F, C), m.randn(F)
    f = gc.gc_linear(X, W, b, _code(gc, act), z=True)
    out = gc.gc_linear_backward(dy, X, W, N, n_c, z=f["z"], act=_code(gc, act))
    at = lambda X, W, b: (gc.gc_linear(X, W, b, _code(gc, act))["y"].double() * dy).view(N, -1).sum(1)
    t = 2.0 ** -7
    diff = lambda dX, dW, db: (at(X + t * dX, W + t * dW, b + t * db) - at(X - t * dX, W - t * dW, b - t * db)) / (2 * t)
    o = 0.0
    assert abs(diff(s, o, o).sum() - (out["dx"].double() * s).sum()).item() <= 0.1
    assert (diff(o, q, o) - out["G"].double() @ q.double().flatten()).abs().max().item() <= 0.1
    assert (diff(o, o, r) - out["Gb"].double() @ r.double()).abs().max().item() <= 0.1


@pytest.mark.parametrize("x,n_c", [("f32", 5569), ("bf16", 8000)])
def test_long_sums_keep_their_digits(gc, x, n_c):
    """fp32 sums over thousands of points or columns, in the 2-norm: at most 48 additions in a row in tensor memory, each
    cut off by 2^-24 of a running sum of two thirds on average: 1.9e-6, and the operands 2^-18 on average with bf16's hi + lo,
    3.8e-6: 6e-6 together."""
    m = Maker(n_c)
    C, F = 136, 300
    X, W, z, dy = m.mat(n_c, C, TYPES[x]), m.mat(F, C, TYPES[x]), m.mat(n_c, F, TYPES[x]), m.mat(n_c, F, TYPES[x])
    got = gc.gc_linear_backward(dy, X, W, 1, n_c, z=z, act=gc.GC_ACT_GELU)
    ref = _ref_grad(dy, z, X, W, "gelu", 1)
    for k in ("G", "Gb"):
        assert ((got[k].double() - ref[k][0]).norm() / ref[k][0].norm()).item() <= 6e-6, k
    if x == "f32":
        A, B = m.mat(100, n_c, torch.float32), m.mat(200, n_c, torch.float32)
        want = A.double() @ B.double().T
        assert ((gc.gc_linear(A, B)["y"].double() - want).norm() / want.norm()).item() <= 6e-6


def test_large(gc):
    """More rows than a wave of tiles, a residual in place, offsets past 2^31 bytes in G."""
    m = Maker(17)
    X, W, b = m.mat(9001, 520, torch.bfloat16), m.mat(1030, 520, torch.bfloat16, 0.05), m.randn(1030)
    ws = gc.Workspace()
    got = gc.gc_linear(X, W, b, gc.GC_ACT_SILU, z=True, ws=ws)
    gc.gc_status(ws)
    ref = _ref_linear(X, W, b, "silu", None)
    _close(got["y"], ref["y"], "y")
    _close(got["z"], ref["z"], "z")
    N, n_c, C, F = 30, 5, 4100, 4500
    X, W, dy = m.mat(N * n_c, C, torch.bfloat16), m.mat(F, C, torch.bfloat16, 0.02), m.mat(N * n_c, F, torch.bfloat16)
    G = gc.gc_linear_backward(dy, X, W, N, n_c, dx=False, Gb=False)["G"]
    for i in (0, 29):
        r = slice(i * n_c, (i + 1) * n_c)
        want, S = dy[r].double().T @ X[r].double(), dy[r].double().abs().T @ X[r].double().abs()
        assert ((G[i].view(F, C).double() - want).abs() <= 40 * 2.0 ** -23 * S).all()


def test_on_another_stream_and_in_a_graph(gc):
    m = Maker(12)
    N, n_c, C, F = 2, 64, 136, 700
    X, W, dy = m.mat(N * n_c, C, torch.bfloat16), m.mat(F, C, torch.float32), m.mat(N * n_c, F, torch.bfloat16)
    f = gc.gc_linear(X * 2, W, act=gc.GC_ACT_GELU, z=True)
    want = gc.gc_linear_backward(dy * 2, X * 2, W, N, n_c, z=f["z"], act=gc.GC_ACT_GELU)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    ws = gc.Workspace()
    with torch.cuda.stream(s):
        X2, dy2 = X * 2, dy * 2
        got = gc.gc_linear(X2, W, act=gc.GC_ACT_GELU, z=True, ws=ws)
        back = gc.gc_linear_backward(dy2, X2, W, N, n_c, z=got["z"], act=gc.GC_ACT_GELU, ws=ws)
    s.synchronize()
    assert all(torch.equal(got[k], f[k]) for k in f) and all(torch.equal(back[k], want[k]) for k in want)
    for t in (*got.values(), *back.values()):
        t.zero_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        gc.gc_linear(X2, W, act=gc.GC_ACT_GELU, y=got["y"], z=got["z"], ws=ws)
        gc.gc_linear_backward(dy2, X2, W, N, n_c, z=got["z"], act=gc.GC_ACT_GELU, ws=ws, **back)
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(got[k], f[k]) for k in f) and all(torch.equal(back[k], want[k]) for k in want)
    gc.gc_status(ws)


@pytest.mark.parametrize("backward", [False, True])
def test_stall_times_out_then_recovers(gc, backward):
    """The failure path without a fault: the loads are withheld, the waits expire, the status says so and the next call is
    right."""
    m = Maker(14)
    X, W, dy = m.mat(300, 256, torch.bfloat16), m.mat(1500, 256, torch.bfloat16), m.mat(300, 1500, torch.bfloat16)
    ws = gc.Workspace()

    def call():
        if backward:
            return gc.gc_linear_backward(dy, X, W, 2, 150, Gb=False, ws=ws)
        return gc.gc_linear(X, W, z=True, ws=ws)
    want = call()
    gc.gc_set_wait_limit(1 << 22)
    try:
        gc.gc_inject_stall(gc.GC_STALL_LINEAR)
        call()
        torch.cuda.synchronize()
        with pytest.raises(gc.GCError) as e:
            gc.gc_status(ws)
        assert e.value.code == -5
    finally:
        gc.gc_inject_stall(0)
        gc.gc_set_wait_limit(0)
    got = call()
    gc.gc_status(ws)
    assert all(torch.equal(got[k], want[k]) for k in want if want[k] is not None)
