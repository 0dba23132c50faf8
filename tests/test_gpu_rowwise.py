"""gc_dropout, gc_layer_norm and gc_layer_norm_backward against the fp64 oracle.

Tolerances, with u = 2^-24 (a rounding to fp32) and v = the rounding of the stored type (u or 2^-8):
sums run over at most 64 fp32 roundings in a chain (32 values a lane, ten tree levels, a few
products), so a mean of h is off by 64 u max|h|, and what is formed from it as stated below; what is
stored is off by v more."""
import numpy as np
import pytest
import torch

from oracle import lm_oracle as L

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
V = {"f32": U, "bf16": 2.0 ** -8}


@pytest.fixture(scope="module")
def gc():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2405_19509_gb300 as m
    return m


def _np(t):
    return t.double().cpu().numpy()


def _mat(rng, rows, cols, dtype, layout="dense", scale=1.0, shift=0.0):
    """A CUDA matrix: dense, with rows apart, or with rows apart off every 16-byte boundary."""
    a = torch.from_numpy((scale * rng.standard_normal((rows, cols)) + shift).astype(np.float32)).to(TYPES[dtype]).cuda()
    if layout == "dense":
        return a
    pad, first = (8, 8) if layout == "strided" else (5, 3)
    big = torch.full((rows, cols + pad + first), float("nan"), dtype=a.dtype, device="cuda")
    big[:, first:first + cols] = a
    return big[:, first:first + cols]


def _like(t, layout):
    """An output of t's shape in the layout, and the whole buffer with its sentinel value."""
    rows, cols = t.shape
    pad, first = {"dense": (0, 0), "strided": (8, 8), "ragged": (5, 3)}[layout]
    big = torch.full((rows, cols + pad + first), -77.0, dtype=t.dtype, device="cuda")
    return big[:, first:first + cols], big


def _untouched(big, view):
    first = view.storage_offset()
    keep = torch.ones(big.shape[1], dtype=torch.bool)
    keep[first:first + view.shape[1]] = False
    assert (big[:, keep.cuda()] == -77.0).all()


# ------------------------------------------------------------------------------------ dropout
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("layout", ["dense", "strided", "ragged"])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 8), (3, 7), (2, 255), (5, 256), (4, 264), (3, 1001)])
def test_dropout_matches_oracle(gc, dtype, layout, rows, cols):
    rng = np.random.default_rng(rows * 1000 + cols)
    x, r = _mat(rng, rows, cols, dtype, layout), _mat(rng, rows, cols, dtype, layout)
    seed, offset, row0 = 0xFEDCBA9876543210, (5 << 32) + 7, (1 << 33) + 3
    for p, res in ((0.0, r), (0.1, None), (0.5, r), (0.99999, None)):
        out, big = _like(x, layout)
        got = gc.gc_dropout(x, p, seed, offset, row0, residual=res, out=out)
        assert got is out
        _untouched(big, out)
        ref = L.dropout(_np(x), p, seed, offset, row0, None if res is None else _np(res))
        mag = np.abs(L.dropout(np.abs(_np(x)), p, seed, offset, row0)) + (0 if res is None else np.abs(_np(res)))
        # the scale, the product and the sum round, then the store
        assert (np.abs(_np(out) - ref) <= 3 * U * mag + V[dtype] * np.abs(ref)).all()
        if p and res is None:
            assert np.array_equal(_np(out) != 0, (ref != 0))


def test_dropout_mask_does_not_depend_on_the_call(gc):
    """The same points draw the same mask in fp32 and bf16, whole or in parts, in any layout."""
    rng = np.random.default_rng(5)
    ones = torch.ones(64, 520, device="cuda")
    whole = gc.gc_dropout(ones, 0.3, 11, 4)
    assert torch.equal(gc.gc_dropout(ones.bfloat16(), 0.3, 11, 4) != 0, whole != 0)
    assert torch.equal(gc.gc_dropout(ones[:8], 0.3, 11, 4, row0=40), whole[40:48])
    odd = torch.ones(64, 523, device="cuda")[:, 3:]
    assert torch.equal(gc.gc_dropout(odd, 0.3, 11, 4), whole)
    assert not torch.equal(gc.gc_dropout(ones, 0.3, 12, 4), whole)
    assert not torch.equal(gc.gc_dropout(ones, 0.3, 11, 5), whole)
    big = gc.gc_dropout(torch.ones(4096, 1024, device="cuda"), 0.3, 1, 1)
    t = L.drop_threshold(0.3) / 65536
    n = big.numel()
    assert abs((big == 0).sum().item() / n - t) <= 6 * (t * (1 - t) / n) ** 0.5


def test_dropped_values_are_zero_whatever_they_hold(gc):
    x = torch.full((4, 1000), float("nan"), device="cuda")
    x[1] = float("inf")
    r = torch.randn(4, 1000, device="cuda")
    out = gc.gc_dropout(x, 0.5, 3, 1, residual=r)
    keep = torch.from_numpy(L.keep_mask(4, 1000, 0.5, 3, 1)).cuda()
    assert torch.equal(out[~keep], r[~keep])
    assert not torch.isfinite(out[keep]).any()


def test_dropout_in_place_and_empty(gc):
    x = torch.randn(300, 777, device="cuda")
    r = torch.randn_like(x)
    ref = gc.gc_dropout(x, 0.2, 1, 2, residual=r)
    a, b = x.clone(), r.clone()
    assert torch.equal(gc.gc_dropout(a, 0.2, 1, 2, residual=r, out=a), ref)
    assert torch.equal(gc.gc_dropout(x, 0.2, 1, 2, residual=b, out=b), ref)
    n = gc.gc_kernel_launches()
    assert gc.gc_dropout(x[:0], 0.2, 1).shape == (0, 777)
    assert gc.gc_kernel_launches() == n


def test_rows_past_32_bit_offsets(gc):
    """Rows 2^31 elements apart: every byte offset of the last ones is past 32 bits."""
    buf = torch.zeros((1 << 32) + 4096, dtype=torch.bfloat16, device="cuda")
    x = torch.as_strided(buf, (3, 512), (1 << 31, 1))
    src = torch.randn(3, 512, device="cuda").bfloat16()
    x.copy_(src)
    assert torch.equal(gc.gc_dropout(x, 0.25, 4, 4), gc.gc_dropout(src, 0.25, 4, 4))
    a, b = gc.gc_layer_norm(x), gc.gc_layer_norm(src)
    assert torch.equal(a["y"], b["y"]) and torch.equal(a["rstd"], b["rstd"])
    g, h = (gc.gc_layer_norm_backward(src, t, b["mean"], b["rstd"], None, 1, 3, dx=o)
            for t, o in ((x, x), (src, True)))
    assert torch.equal(g["dx"], h["dx"]) and torch.equal(g["G"], h["G"])


# ------------------------------------------------------------------------------------ layer norm
SHAPES = [(1, 1), (2, 2), (3, 7), (1, 256), (5, 255), (4, 300), (3, 512), (200, 1000), (2, 1024),
          (3, 1025), (160, 2048), (2, 4096), (155, 3001), (153, 4096), (2, 5000), (153, 8192), (1, 8200),
          (2, 20001), (1, 32768)]


def _norm_ref(x, r, p, seed, offset, row0, gamma, beta, eps):
    h = L.dropout(_np(x), p, seed, offset, row0, None if r is None else _np(r))
    return (h,) + L.layer_norm(h, gamma, beta, eps)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("layout", ["dense", "ragged"])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_layer_norm_matches_oracle(gc, dtype, layout, rows, cols):
    rng = np.random.default_rng(rows * 7 + cols)
    x = _mat(rng, rows, cols, dtype, layout, 2.0, 3.0)
    small = rows * cols < 40000          # the oracle draws masks in Python
    p = 0.2 if small else 0.0
    r = _mat(rng, rows, cols, dtype, layout) if cols % 2 else None
    g = 1 + 0.3 * rng.standard_normal(cols)
    b = rng.standard_normal(cols)
    gt, bt = (torch.from_numpy(v.astype(np.float32)).cuda() for v in (g, b))
    g, b = _np(gt), _np(bt)
    eps = 1e-5
    y, big = _like(x, layout)
    hbuf, hbig = _like(x, layout)
    got = gc.gc_layer_norm(x, gt, bt, eps, residual=r, p=p, seed=5, offset=9, row0=17, y=y, h=hbuf)
    _untouched(big, y)
    _untouched(hbig, hbuf)
    h, ref, mean, rstd = _norm_ref(x, r, p, 5, 9, 17, g, b, eps)
    top = np.abs(h).max(1)
    # h itself: scale, product and sum
    assert (np.abs(_np(got["h"]) - h) <= 3 * U * (np.abs(h) + 4 * top[:, None]) + V[dtype] * np.abs(h)).all()
    off = 70 * U * top                                        # of the mean, and of h - mean
    assert (np.abs(_np(got["mean"]) - mean) <= off).all()
    # the variance is off by 64 u of itself and 2 off times the spread; rstd by half as much, relatively
    rel = 40 * U + 2 * off * rstd
    assert (np.abs(_np(got["rstd"]) - rstd) <= rel * rstd).all()
    tol = (2 * off * rstd)[:, None] * np.abs(g) + (rel[:, None] + 4 * U) * np.abs(ref - b) + 2 * U * np.abs(b)
    assert (np.abs(_np(y) - ref) <= tol + V[dtype] * np.abs(ref)).all()


def test_layer_norm_of_far_means_and_constant_rows(gc):
    """A mean 2^12 times the spread keeps the spread's digits; a constant row gives beta."""
    rng = np.random.default_rng(3)
    for cols in (100, 1000, 4096, 9000):
        x = _mat(rng, 200, cols, "f32", "dense", 1.0, 4096.0)
        x[7] = 1.25
        b = torch.randn(cols, device="cuda")
        y = gc.gc_layer_norm(x, None, b, 1e-5)
        _, ref, mean, rstd = _norm_ref(x, None, 0, 0, 0, 0, 1.0, _np(b), 1e-5)
        # the mean is off by 70 u 4100; y by that times rstd
        live = np.arange(200) != 7
        assert (np.abs(_np(y["y"]) - ref)[live] <= 2 * 70 * U * 4100 * rstd[live, None] + 1e-3 * 0.01).all()
        assert torch.equal(y["y"][7], b) and y["mean"][7] == 1.25


def test_layer_norm_defaults_and_nonfinite_rows(gc):
    x = torch.randn(6, 700, device="cuda")
    ref = gc.gc_layer_norm(x)
    bad = x.clone()
    bad[2, 699] = float("nan")
    bad[4, 0] = float("inf")
    got = gc.gc_layer_norm(bad, mean=False, rstd=False)
    live = [0, 1, 3, 5]
    assert torch.equal(got["y"][live], ref["y"][live]) and got["mean"] is None
    assert not torch.isfinite(got["y"][[2, 4]]).any()
    assert ref["h"] is x
    # in place: y over x, h over residual
    r = torch.randn_like(x)
    want = gc.gc_layer_norm(x, residual=r, p=0.1, seed=1)
    x2, r2 = x.clone(), r.clone()
    got = gc.gc_layer_norm(x2, residual=r2, p=0.1, seed=1, y=x2, h=r2)
    assert torch.equal(x2, want["y"]) and torch.equal(r2, want["h"])
    assert gc.gc_layer_norm(x[:0])["y"].shape == (0, 700)


# ------------------------------------------------------------------------------------ its gradient
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("layout", ["dense", "ragged"])
@pytest.mark.parametrize("N,n_c,cols", [(1, 1, 1), (1, 1, 8), (3, 5, 7), (6, 32, 64), (2, 77, 250), (1, 300, 256),
                                        (2, 33, 500), (3, 9, 512), (2, 10, 1000), (20, 7, 1001), (1, 200, 2048),
                                        (2, 3, 3000), (1, 40, 4096), (2, 5, 8192), (2, 70, 8200), (1, 3, 32768)])
def test_layer_norm_backward_matches_oracle(gc, dtype, layout, N, n_c, cols):
    rng = np.random.default_rng(N * 100 + n_c + cols)
    rows = N * n_c
    h = _mat(rng, rows, cols, dtype, layout, 1.5, 0.5)
    dy, dh = _mat(rng, rows, cols, dtype, layout), _mat(rng, rows, cols, dtype, layout)
    gt = torch.from_numpy((1 + 0.3 * rng.standard_normal(cols)).astype(np.float32)).cuda()
    f = gc.gc_layer_norm(h, gt, None, 1e-5)
    p = 0.2 if rows * cols < 40000 else 0.0
    dx, bx = _like(dy, layout)
    dr, br = _like(dy, layout)
    wide = torch.full((N, 2 * cols + 9), -77.0, device="cuda")     # a slice of a model's chunk gradients
    G = wide[:, 4:4 + 2 * cols]
    ws = gc.Workspace()
    gc.gc_layer_norm_backward(dy, h, f["mean"], f["rstd"], gt, N, n_c, dh=dh, p=p, seed=8, offset=1, row0=2,
                              dx=dx, dresidual=dr, G=G, ws=ws)
    gc.gc_status(ws)
    for big, view in ((bx, dx), (br, dr)):
        _untouched(big, view)
    assert (wide[:, :4] == -77).all() and (wide[:, 4 + 2 * cols:] == -77).all()
    mean, rstd, g = _np(f["mean"]), _np(f["rstd"]), _np(gt)
    d, Gr = L.layer_norm_grad(_np(dy), _np(h), mean, rstd, g, N)
    ref = d + _np(dh)
    # n is off by 3 u (|h| + |mean|) rstd; the two means by 64 u of their terms' size and n's error
    a = np.abs(_np(dy) * g)
    n = np.abs((_np(h) - mean[:, None]) * rstd[:, None])
    dn = 3 * U * (np.abs(_np(h)) + np.abs(mean)[:, None]) * rstd[:, None]
    m1, m2, e2 = a.mean(1, keepdims=True), (a * n).mean(1, keepdims=True), (a * dn).mean(1, keepdims=True)
    tol = rstd[:, None] * (70 * U * (a + m1 + n * m2) + dn * m2 + n * e2) + 4 * U * (np.abs(d) + np.abs(ref))
    assert (np.abs(_np(dr) - ref) <= tol + V[dtype] * np.abs(ref)).all()
    refx = L.dropout(ref, p, 8, 1, 2)
    assert (np.abs(_np(dx) - refx) <= 1.5 * tol + (2 * U + V[dtype]) * np.abs(refx)).all()
    # a column's sum over a chunk: at most n_c + 16 roundings, and n's error
    ady = np.abs(_np(dy)).reshape(N, n_c, cols)
    tg = (n_c + 16) * U * (ady * n.reshape(N, n_c, cols)).sum(1) + (ady * dn.reshape(N, n_c, cols)).sum(1)
    tb = (n_c + 16) * U * ady.sum(1)
    assert (np.abs(_np(G) - Gr) <= np.concatenate([tg, tb], 1) + 1e-30).all()


def test_layer_norm_backward_outputs_alone_in_place_and_repeated(gc):
    """Each output alone is the same output of the full call (values below 5: 70 u of a few of them);
    gradients may be written over their inputs; a second call gives the same bits."""
    N, n_c = 3, 50
    for cols in (96, 1000, 4096, 10000):
        dy, h, dh = (torch.randn(N * n_c, cols, device="cuda") for _ in range(3))
        f = gc.gc_layer_norm(h)
        ws = gc.Workspace()
        run = lambda **k: gc.gc_layer_norm_backward(dy, h, f["mean"], f["rstd"], None, N, n_c, p=0.1, seed=1,
                                                    ws=ws, **{"dh": dh, **k})
        full = run(dresidual=True)
        again = run(dresidual=True)
        assert all(torch.equal(full[k], again[k]) for k in full)
        assert torch.allclose(run(dx=False)["G"], full["G"], rtol=1e-5, atol=2e-5)
        assert torch.allclose(run(G=False)["dx"], full["dx"], rtol=1e-5, atol=2e-5)
        only = run(G=False, dx=False, dresidual=True)
        assert only["G"] is None and torch.allclose(only["dresidual"], full["dresidual"], rtol=1e-5, atol=2e-5)
        a, b = dy.clone(), dh.clone()
        got = gc.gc_layer_norm_backward(a, h, f["mean"], f["rstd"], None, N, n_c, dh=b, p=0.1, seed=1, dx=a,
                                        dresidual=b, ws=ws)
        assert torch.equal(a, full["dx"]) and torch.equal(b, full["dresidual"]) and torch.equal(got["G"], full["G"])


def test_layer_norm_gradient_against_differences_of_the_forward(gc):
    """d/dt of sum(dy * y(x + t s)) by central differences of the GPU's own forward pass.  In fp32 a
    value of y is off by about 4 u |y|; the sum of 3,000 of them by sqrt(3000) times that, over 2 t
    with t = 2^-5, and the cubic term is t^2 of a third derivative of order |dy| rstd^3: 2e-2 of a
    derivative of order sqrt(3000)."""
    N, n_c, cols = 2, 5, 300
    g = torch.Generator(device="cuda").manual_seed(4)
    x, r, dy, s = (torch.randn(N * n_c, cols, device="cuda", generator=g) for _ in range(4))
    gamma = 1 + 0.2 * torch.randn(cols, device="cuda", generator=g)
    kw = dict(p=0.25, seed=6, offset=2)
    f = gc.gc_layer_norm(x, gamma, None, residual=r, **kw)
    b = gc.gc_layer_norm_backward(dy, f["h"], f["mean"], f["rstd"], gamma, N, n_c, dresidual=True, **kw)
    t = 2.0 ** -5
    total = lambda a, c, gm: (gc.gc_layer_norm(a, gm, None, residual=c, **kw)["y"].double() * dy.double()).sum().item()
    for lo, hi, want in ((total(x - t * s, r, gamma), total(x + t * s, r, gamma), (b["dx"].double() * s).sum()),
                         (total(x, r - t * s, gamma), total(x, r + t * s, gamma), (b["dresidual"].double() * s).sum()),
                         (total(x, r, gamma - t * s[0]), total(x, r, gamma + t * s[0]),
                          (b["G"][:, :cols].double().sum(0) * s[0]).sum())):
        assert abs((hi - lo) / (2 * t) - want.item()) <= 2e-2 * 3000 ** 0.5


def test_rowwise_on_another_stream(gc):
    """Calls run on torch's current stream: work queued there before them is seen."""
    s = torch.cuda.Stream()
    x = torch.randn(2000, 1024, device="cuda")
    want = gc.gc_layer_norm(x + 1)["y"]
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        got = gc.gc_layer_norm(x + 1)["y"]
        out = gc.gc_dropout(got, 0.0, 1)
    s.synchronize()
    assert torch.equal(got, want) and torch.equal(out, want)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("cols", [256, 1001, 9000])
def test_layer_norm_over_its_input_gives_what_the_gradient_takes(gc, dtype, cols):
    """y written over x, nothing else asked for: h is x as it was."""
    rng = np.random.default_rng(cols)
    x = _mat(rng, 12, cols, dtype, "strided")
    before = x.clone()
    want = gc.gc_layer_norm(before)
    f = gc.gc_layer_norm(x, y=x)
    assert f["y"] is x and torch.equal(x, want["y"]) and torch.equal(f["h"], before)
    dy = _mat(rng, 12, cols, dtype)
    a = gc.gc_layer_norm_backward(dy, want["h"], want["mean"], want["rstd"], None, 3, 4)
    b = gc.gc_layer_norm_backward(dy, f["h"], f["mean"], f["rstd"], None, 3, 4)
    assert torch.equal(a["dx"], b["dx"]) and torch.equal(a["G"], b["G"])


def test_layer_norm_backward_of_as_many_rows_as_there_may_be(gc):
    """A chunk of 2^31 - 1 rows of one column, whose last slice ends past 32 bits.  Every row adds 1 to the
    gradient of beta and 2^-10 to gamma's.  Chains of fewer than 2^24 additions of ones are exact, the
    sums of at most 2^12 slices round by 2^-24 each: 2^-12 of the total."""
    rows = (1 << 31) - 1
    one = torch.ones(rows, 1, dtype=torch.bfloat16, device="cuda")
    stat = torch.full((rows,), 2.0 ** -5, device="cuda")
    h = torch.full((rows, 1), 2.0 ** -4, dtype=torch.bfloat16, device="cuda")
    G = gc.gc_layer_norm_backward(one, h, stat, stat, None, 1, rows, dx=False)["G"].double()
    assert abs(G[0, 1].item() / rows - 1) <= 2.0 ** -12 and abs(G[0, 0].item() * 2.0 ** 10 / rows - 1) <= 2.0 ** -12
    del one, stat, h
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("cols", [33, 40, 264, 1000, 1001, 8185, 8200])
def test_gradient_of_constant_rows_of_large_values(gc, dtype, cols):
    """Rows of 2^110 and a reciprocal deviation of 2^20, whose product is past fp32's range: n is zero, and
    dx = rstd (a - mean a).  64 roundings a sum, as many in dx, and the store."""
    rng = np.random.default_rng(cols)
    dy = _mat(rng, 6, cols, dtype)
    h = torch.full((6, cols), 2.0 ** 110, dtype=dy.dtype, device="cuda")
    mean, rstd = torch.full((6,), 2.0 ** 110, device="cuda"), torch.full((6,), 2.0 ** 20, device="cuda")
    got = gc.gc_layer_norm_backward(dy, h, mean, rstd, None, 2, 3)
    a = _np(dy)
    want = 2.0 ** 20 * (a - a.mean(1, keepdims=True))
    assert (np.abs(_np(got["dx"]) - want) <= 2.0 ** 20 * 70 * U * np.abs(a).max() + V[dtype] * np.abs(want)).all()
    G = _np(got["G"])
    assert not G[:, :cols].any() and (np.abs(G[:, cols:] - a.reshape(2, 3, cols).sum(1)) <= 4 * U * 3 * np.abs(a).max()).all()
