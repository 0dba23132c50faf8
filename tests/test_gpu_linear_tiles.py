"""gc_linear and gc_linear_backward where tiles on the tensor cores take the work: digits of their results, values that are
not finite or at the end of the range, outputs over inputs, graphs.  Every test asserts that its sizes reach the tiles."""
import pytest
import torch

from test_gpu_linear import PAIRS, TYPES, Maker, _act, _close, _code, _ref_grad, _ref_linear, _untouched, gc  # noqa: F401

pytestmark = pytest.mark.gpu


def _t(dtype):
    return 1 if dtype == torch.bfloat16 else 0


def _by_tiles(gc, T, C, F, x, w, joined=None):
    """Copies of rows on no boundary take a workspace on the tiles' path alone; of rows on one, ranges of a sum do."""
    assert T > 8 and gc.lib.gc_linear_workspace(T, C, F, _t(TYPES[x]), _t(TYPES[w]), 0, 0) > 256
    if joined is not None:
        assert x == w == "bf16" and (gc.lib.gc_linear_workspace(T, C, F, 1, 1, 1, 1) > 256) == joined


def _back_by_tiles(gc, N, n_c, C, F, x, w, want=3):
    for k in (1, 2):
        assert not want & k or gc.lib.gc_linear_backward_workspace(N, n_c, C, F, _t(TYPES[x]), _t(TYPES[w]), 2, 0, 0, 0, k) > 256


def _norm_off(got, ref):
    return ((got.double() - ref).norm() / ref.norm()).item()


GRADS = [(2, 150, 520, 1000), (4, 77, 1000, 1031), (1, 700, 264, 4000), (8, 256, 512, 2048)]


@pytest.mark.parametrize("act", ["gelu", "silu", "relu", "none"])
@pytest.mark.parametrize("w", ["bf16", "f32"])
@pytest.mark.parametrize("N,n_c,C,F", GRADS)
def test_dx_of_bf16_rows_is_rounded_once(gc, N, n_c, C, F, w, act):
    """dx of bf16 rows is the fp32 product's, rounded: a value v off by e before it is rounded ends at most 2 e further from v
    than v's own rounding.  e in the 2-norm, of terms of either sign: d and W as hi + lo, 2^-18 each and 2^-18 for lo lo, the
    slope 2^-19; 2 F / 16 (with an fp32 W 3 F / 16) additions cut off by 2^-24 of a running sum of two thirds."""
    _back_by_tiles(gc, N, n_c, C, F, "bf16", w, 1)
    m = Maker(N + F)
    T = N * n_c
    X, W, z, dy = m.mat(T, C, torch.bfloat16), m.mat(F, C, TYPES[w], C ** -0.5), m.mat(T, F, torch.bfloat16, 1.5), m.mat(T, F, torch.bfloat16)
    ref = _ref_grad(dy, z, X, W, act, N)["dx"][0]
    e = 3 * 2.0 ** -18 + 2.0 ** -19 + (3 if w == "f32" else 2) * F / 16 * 2 / 3 * 2.0 ** -24
    once = _norm_off(ref.to(torch.bfloat16), ref)
    for G in (True, False):
        got = gc.gc_linear_backward(dy, X, W, N, n_c, z=z, act=_code(gc, act), G=G, Gb=False)["dx"]
        assert _norm_off(got, ref) <= once + 2 * e


@pytest.mark.parametrize("act", ["gelu", "gelu_tanh", "silu", "relu", "none"])
@pytest.mark.parametrize("N,n_c,C,F", GRADS)
def test_G_of_bf16_rows_keeps_fp32_digits(gc, N, n_c, C, F, act):
    """G is an fp32 result: of bf16 rows in the 2-norm at most 48 additions in a row, each cut off by 2^-24 of a running sum of
    two thirds, 1.9e-6, and the slope 2^-22 on average (2^-19 at its worst): 2.1e-6.  d as hi + lo would add 2^-18 to 2^-17."""
    _back_by_tiles(gc, N, n_c, C, F, "bf16", "bf16", 2)
    m = Maker(N + C)
    T = N * n_c
    X, W, z, dy = m.mat(T, C, torch.bfloat16), m.mat(F, C, torch.bfloat16), m.mat(T, F, torch.bfloat16), m.mat(T, F, torch.bfloat16)
    got = gc.gc_linear_backward(dy, X, W, N, n_c, z=z, act=_code(gc, act), dx=False)
    ref = _ref_grad(dy, z, X, W, act, N)
    for k in ("G", "Gb"):
        assert _norm_off(got[k], ref[k][0]) <= 2.1e-6, k


@pytest.mark.parametrize("T,C,F", [(2048, 64, 1024), (1024, 128, 1031), (700, 520, 1000), (300, 4100, 520), (129, 8192, 136)])
def test_fp32_rows_keep_fp32_digits(gc, T, C, F):
    """fp32 rows enter as three parts, 24 bits.  At most 28 additions in a row meet a sum of its full size, each cut off by 2^-24 of
    a running sum of two thirds, 1.1e-6, and the products left out 2^-24, the parts 2^-26: 1.2e-6, and of one K block of 64, where
    four are of full size, 0.16e-6 + 0.07e-6.  Two parts would be 4.4e-6 off, 48 additions 1.9e-6."""
    _by_tiles(gc, T, C, F, "f32", "f32")
    m = Maker(C)
    X, W = m.mat(T, C, torch.float32), m.mat(F, C, torch.float32, C ** -0.5)
    got = gc.gc_linear(X, W)["y"]
    assert _norm_off(got, X.double() @ W.double().T) <= (0.25e-6 if C == 64 else 0.8e-6)


@pytest.mark.parametrize("x,act", [("f32", "gelu"), ("f32", "none"), ("bf16", "gelu"), ("bf16", "none")])
@pytest.mark.parametrize("N,n_c,C,F", GRADS + [(3, 64, 520, 1000), (1, 5000, 136, 300)])
def test_fp32_sums_of_chunks_keep_fp32_digits(gc, N, n_c, C, F, x, act):
    """At most 28 additions of full size in a row (24 of bf16 products): 1.1e-6 at the most as above, all at their worst; a cut
    is half of 2^-24 on average: 0.6e-6, and 0.2e-6 for d, the products left out and the joins."""
    _back_by_tiles(gc, N, n_c, C, F, x, x)
    m = Maker(N + F)
    T = N * n_c
    X, W, z, dy = m.mat(T, C, TYPES[x]), m.mat(F, C, TYPES[x], C ** -0.5), m.mat(T, F, TYPES[x]), m.mat(T, F, TYPES[x])
    got = gc.gc_linear_backward(dy, X, W, N, n_c, z=z, act=_code(gc, act))
    ref = _ref_grad(dy, z, X, W, act, N)
    for k in ("dx", "G", "Gb") if x == "f32" else ("G", "Gb"):
        assert _norm_off(got[k], ref[k][0]) <= 0.8e-6, k


@pytest.mark.parametrize("act", ["gelu", "gelu_tanh", "silu", "relu"])
@pytest.mark.parametrize("T,C,F,tiles", [(5, 64, 40, False), (40, 64, 40, False), (1024, 64, 1024, True), (1024, 64, 1021, True)])
def test_activations_far_from_zero(gc, T, C, F, tiles, act):
    """z is the row's first value alone.  act(+inf) is +inf, act(-inf) what its formula gives, far values are themselves or 0, and
    a row's do not reach the next."""
    if tiles:
        _by_tiles(gc, T, C, F, "bf16", "bf16")
    bf = torch.bfloat16
    far = torch.tensor([float("inf"), float("-inf"), float("nan"), 3e38, -3e38, 1e19, -1e19, 200.0, -200.0, 0.0, 40.0, -40.0, 1.0], device="cuda").to(bf)
    X, W = torch.zeros(T, C, device="cuda", dtype=bf), torch.zeros(F, C, device="cuda", dtype=bf)
    X[:, 0] = far[torch.arange(T, device="cuda") % len(far)]
    W[:, 0] = 1.0
    got = gc.gc_linear(X, W, act=_code(gc, act), z=True)
    v = X[:, :1].double()
    want = _act(v, act).expand(T, F)
    if act == "gelu":
        want = torch.where(v == float("-inf"), float("nan"), want)       # -inf times 0, as the others'
    assert torch.equal(got["z"].isnan(), v.isnan().expand(T, F)) and torch.equal(got["z"].isinf(), v.isinf().expand(T, F))
    assert torch.equal(got["y"].isnan(), want.isnan().contiguous())
    assert torch.allclose(got["y"].double(), want, rtol=2.0 ** -7, atol=1e-30, equal_nan=True)


@pytest.mark.parametrize("x,w", PAIRS)
@pytest.mark.parametrize("layout", ["dense", "ragged"])
def test_a_row_reaches_its_own_alone(gc, x, w, layout):
    """Infinities and NaN in one row of x or of dy, with tiles and with ranges joined: the other rows keep their bits."""
    for T, C, F, joined in ((300, 520, 1000, None), (300, 4096, 264, True)):
        if joined is None or layout == "dense" and x == w == "bf16":
            _by_tiles(gc, T, C, F, x, w, joined)
        _back_by_tiles(gc, 2, T // 2, C, F, x, w)
        m = Maker(T + C, layout)
        t = TYPES[x]
        X, W, z, dy = m.mat(T, C, t), m.mat(F, C, TYPES[w]), m.mat(T, F, t), m.mat(T, F, t)
        want = gc.gc_linear(X, W, act=gc.GC_ACT_RELU, z=True)
        back = gc.gc_linear_backward(dy, X, W, 2, T // 2, z=z, act=gc.GC_ACT_GELU)
        rest = torch.arange(T, device="cuda") != 1
        for bad in (float("inf"), float("-inf"), float("nan")):
            X2, dy2 = X.clone(), dy.clone()
            X2[1, 3] = bad
            dy2[1, 7] = bad
            got = gc.gc_linear(X2, W, act=gc.GC_ACT_RELU, z=True)
            assert all(torch.equal(got[k][rest], want[k][rest]) for k in got) and not torch.isfinite(got["z"][1]).any()
            got = gc.gc_linear_backward(dy2, X, W, 2, T // 2, z=z, act=gc.GC_ACT_GELU)
            assert torch.equal(got["dx"][rest], back["dx"][rest]) and not torch.isfinite(got["dx"][1]).any()
            assert torch.equal(got["G"][1], back["G"][1]) and torch.equal(got["Gb"][1], back["Gb"][1])
            assert not torch.isfinite(got["G"][0].view(F, C)[7]).any() and torch.isfinite(got["G"][0].view(F, C)[8:]).all()
            assert not torch.isfinite(got["Gb"][0, 7]) and torch.isfinite(got["Gb"][0, 8:]).all()


@pytest.mark.parametrize("layout", ["dense", "ragged"])
def test_values_at_the_end_of_the_range(gc, layout):
    """fp32's largest values round past bf16's; alone in a row they are themselves in y, dx and G, to 2^-22: three parts that are
    cut off keep 24 bits, their sums are cut off once or twice.  2^-100 times 2^-120 is below fp32's smallest, 2^-149."""
    T, C, F = 300, 520, 1000
    _by_tiles(gc, T, C, F, "f32", "f32")
    _back_by_tiles(gc, 1, T, C, F, "f32", "f32")
    m = Maker(1, layout)
    big = 3.4028234e38
    X, W = m.mat(T, C, torch.float32, 0.0), m.mat(F, C, torch.float32, 0.0)
    X[0, 5], X[1, 6], X[2, 7], X[290, 519] = big, -big, 2.0 ** -120, big
    W[:, 5], W[:, 6], W[:, 7], W[:, 519] = 1.0, 0.5, 1.0, -1.0
    near = lambda got, want: bool(((got.double() - want).abs() <= 2.0 ** -22 * want.abs() + 2.0 ** -149).all())
    assert near(gc.gc_linear(X, W)["y"], X.double() @ W.double().T)
    assert near(gc.gc_linear(W, X)["y"], W.double() @ X.double().T)              # as the weights
    dy = m.mat(T, F, torch.float32, 0.0)
    dy[0, 3], dy[1, 4], dy[2, 5], dy[290, 999] = big, -big, 2.0 ** -100, 1.0
    got = gc.gc_linear_backward(dy, X.clamp(-1, 1), W, 1, T)
    assert near(got["dx"], dy.double() @ W.double())
    assert near(got["G"][0].view(F, C), dy.double().T @ X.clamp(-1, 1).double())
    assert near(gc.gc_linear_backward(dy.clamp(-1, 1), X, W, 1, T)["G"][0].view(F, C), dy.clamp(-1, 1).double().T @ X.double())


def test_weights_at_the_end_of_the_range_beside_bf16_rows(gc):
    T, C, F = 300, 520, 1000
    _by_tiles(gc, T, C, F, "bf16", "f32")
    X, W = torch.zeros(T, C, device="cuda", dtype=torch.bfloat16), torch.zeros(F, C, device="cuda")
    X[0, 5], X[1, 6] = 1.0, 0.5
    W[:, 5], W[:, 6] = 3.38e38, 3.4028234e38
    got = gc.gc_linear(X, W)["y"].double()
    want = X.double() @ W.double().T
    assert bool(((got - want).abs() <= (2.0 ** -8 + 2.0 ** -15) * want.abs()).all())


@pytest.mark.parametrize("x", ["bf16", "f32"])
@pytest.mark.parametrize("T,C,F,joined", [(300, 520, 1000, None), (300, 520, 1001, None), (300, 4096, 264, True), (300, 4096, 261, None),
                                          (2100, 520, 1032, False)])
def test_y_over_the_residual(gc, x, T, C, F, joined):
    """By boxes, by rows on no boundary, and by the join of ranges."""
    _by_tiles(gc, T, C, F, x, x, joined if x == "bf16" else None)
    m = Maker(4)
    X, W, res = m.mat(T, C, TYPES[x]), m.mat(F, C, TYPES[x], C ** -0.5), m.mat(T, F, TYPES[x])
    want = gc.gc_linear(X, W, act=gc.GC_ACT_GELU, residual=res, z=True)
    _close(want["y"], _ref_linear(X, W, None, "gelu", res)["y"], "y")
    got = gc.gc_linear(X, W, act=gc.GC_ACT_GELU, residual=res, y=res, z=True)
    assert got["y"] is res and torch.equal(res, want["y"]) and torch.equal(got["z"], want["z"])


@pytest.mark.parametrize("x,w", PAIRS)
@pytest.mark.parametrize("T,C,F", [(300, 520, 1000), (300, 4096, 264)])
def test_on_another_stream_and_in_a_graph(gc, T, C, F, x, w):
    """Forward and backward by tiles, copies in parts and joins among them, on a stream of their own and replayed."""
    _by_tiles(gc, T, C, F, x, w)
    _back_by_tiles(gc, 2, T // 2, C, F, x, w)
    m = Maker(12)
    X, W, dy = m.mat(T, C, TYPES[x]), m.mat(F, C, TYPES[w]), m.mat(T, F, TYPES[x])
    f = gc.gc_linear(X * 2, W, act=gc.GC_ACT_GELU, z=True)
    want = gc.gc_linear_backward(dy * 2, X * 2, W, 2, T // 2, z=f["z"], act=gc.GC_ACT_GELU)
    torch.cuda.synchronize()
    s, ws = torch.cuda.Stream(), gc.Workspace()
    with torch.cuda.stream(s):
        X2, dy2 = X * 2, dy * 2
        got = gc.gc_linear(X2, W, act=gc.GC_ACT_GELU, z=True, ws=ws)
        back = gc.gc_linear_backward(dy2, X2, W, 2, T // 2, z=got["z"], act=gc.GC_ACT_GELU, ws=ws)
    s.synchronize()
    assert all(torch.equal(got[k], f[k]) for k in f) and all(torch.equal(back[k], want[k]) for k in want)
    for t in (*got.values(), *back.values()):
        t.zero_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        gc.gc_linear(X2, W, act=gc.GC_ACT_GELU, y=got["y"], z=got["z"], ws=ws)
        gc.gc_linear_backward(dy2, X2, W, 2, T // 2, z=got["z"], act=gc.GC_ACT_GELU, ws=ws, **back)
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(got[k], f[k]) for k in f) and all(torch.equal(back[k], want[k]) for k in want)
    gc.gc_status(ws)


def test_slices_of_a_gradient_matrix(gc):
    """G and Gb as a program has them: columns of an N x d matrix of odd d, from an odd one on, which keep the rest."""
    N, n_c, C, F = 3, 120, 264, 1000
    _back_by_tiles(gc, N, n_c, C, F, "bf16", "bf16")
    m = Maker(8)
    X, W, z, dy = (m.mat(*s, torch.bfloat16) for s in ((N * n_c, C), (F, C), (N * n_c, F), (N * n_c, F)))
    want = gc.gc_linear_backward(dy, X, W, N, n_c, z=z, act=gc.GC_ACT_GELU)
    d = 7 + F * C + F + 4
    d += 1 - d % 2
    all_ = torch.full((N, d), -77.0, device="cuda")
    G, Gb = all_[:, 7:7 + F * C], all_[:, 7 + F * C:7 + F * C + F]
    got = gc.gc_linear_backward(dy, X, W, N, n_c, z=z, act=gc.GC_ACT_GELU, G=G, Gb=Gb)
    assert torch.equal(G, want["G"]) and torch.equal(Gb, want["Gb"]) and torch.equal(got["dx"], want["dx"])
    assert bool((all_[:, :7] == -77).all()) and bool((all_[:, 7 + F * C + F:] == -77).all())


@pytest.mark.parametrize("w", ["bf16", "f32"])
def test_long_sums_of_bf16_results_are_not_cut_off(gc, w):
    """Rounding a result to bf16 leaves its size what it is on average, to 2^-9 over the root of 300,000 values: 4e-6.  512 additions in a row
    in tensor memory are each cut off by up to 2^-24 of a running sum whose share grows evenly to all of it: 512 * 2^-24 / 2 = 1.5e-5."""
    T, C, F = 300, 1 << 15, 1000
    _by_tiles(gc, T, C, F, "bf16", w)
    _back_by_tiles(gc, 1, T, F, C, "bf16", w, 1)
    m = Maker(21)
    X, W = m.mat(T, C, torch.bfloat16), m.mat(F, C, TYPES[w], C ** -0.5)
    size = lambda got, ref: abs(((got.double() * ref).sum() / (ref * ref).sum()).item() - 1)
    assert size(gc.gc_linear(X, W)["y"], X.double() @ W.double().T) <= 2e-5
    V, z = m.mat(C, F, TYPES[w], C ** -0.5), m.mat(T, C, torch.bfloat16)
    got = gc.gc_linear_backward(X, X[:, :F], V, 1, T, z=z, act=gc.GC_ACT_GELU, G=False, Gb=False)
    assert size(got["dx"], _ref_grad(X, z, X[:, :F], V, "gelu", 1)["dx"][0]) <= 2e-5
