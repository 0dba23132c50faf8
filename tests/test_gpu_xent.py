"""gc_softmax_xent against 64-bit references.

Tolerances, element by element, with u = 2^-24.  A product's sum over K in tensor memory: K / 16 + 16
additions to fp32, each off by at most 2^-23 of the sum of magnitudes S.  fp32 operands enter as
bf16 hi + lo, off by 2^-17 each, with a dropped term of 2^-16: 2^-15 S together; P enters G off by
2^-17, and a bf16 dX off by 2^-8 (as fp32 W does there).  An error tz of z moves lse by at most
the largest tz and a probability by its size times both; exponentials and logarithms add 2^-20."""
import numpy as np
import pytest
import torch

from oracle import lm_oracle as L

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
V8 = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


@pytest.fixture(scope="module")
def gc():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2405_19509_gb300 as m
    return m


def _data(N, n_c, C, V, x, w, seed, scale=2.0, ignore=0.1, layout="dense"):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def mat(rows, cols, dtype, s):
        a = (s * torch.randn(rows, cols, generator=g, device="cuda")).to(TYPES[dtype])
        if layout == "dense":
            return a
        big = torch.full((rows, cols + (8 if layout == "strided" else 5)), float("nan"), dtype=a.dtype, device="cuda")
        first = 8 if layout == "strided" else 3
        big[:, first:first + cols] = a
        return big[:, first:first + cols]
    X, W = mat(N * n_c, C, x, 1.0), mat(V, C, w, scale / C ** 0.5)
    y = torch.randint(0, V, (N * n_c,), generator=g, device="cuda")
    y[torch.rand(N * n_c, generator=g, device="cuda") < ignore] = -100
    return X, W, y


def _reference(X, W, y, N):
    """Values and tolerances in 64 bits on the GPU: a dict of (value, tolerance)."""
    Xd, Wd = X.double(), W.double()
    T, C = Xd.shape
    V = Wd.shape[0]
    n_c = T // N
    parts = 2.0 ** -15 if X.dtype == torch.float32 or W.dtype == torch.float32 else 0.0
    z = Xd @ Wd.T
    tz = ((C / 16 + 16) * 2.0 ** -23 + parts) * (Xd.abs() @ Wd.abs().T)
    lse = torch.logsumexp(z, 1)
    tl = tz.amax(1) + 2.0 ** -20 * (1 + lse.abs() + z.abs().amax(1))
    live = y >= 0
    at = y.clamp_min(0)[:, None]
    loss = torch.where(live, lse - z.gather(1, at)[:, 0], torch.zeros_like(lse))
    tloss = torch.where(live, tl + tz.gather(1, at)[:, 0], torch.zeros_like(lse))
    p = torch.exp(z - lse[:, None])
    tp = p * (tz + tl[:, None] + 2.0 ** -20) * live[:, None]
    P = p.scatter_add(1, at, torch.full_like(lse, -1.0)[:, None]) * live[:, None]
    aP = P.abs()
    del z, tz, p
    in_dx = 2.0 ** -15 if X.dtype == torch.float32 else 2.0 ** -8 + (2.0 ** -8 if W.dtype == torch.float32 else 0)
    dX = P @ Wd
    tdx = (tp + aP * (in_dx + (V / 16 + 32) * 2.0 ** -23)) @ Wd.abs()
    tdx += V8["f32" if X.dtype == torch.float32 else "bf16"] * dX.abs()
    in_g = 2.0 ** -15 if X.dtype == torch.float32 else 2.0 ** -17
    tp += aP * (in_g + (n_c / 16 + 16) * 2.0 ** -23)
    c = lambda a: a.view(N, n_c, -1)
    G = torch.bmm(c(P).transpose(1, 2), c(Xd)).flatten(1)
    tG = torch.bmm(c(tp).transpose(1, 2), c(Xd.abs())).flatten(1)
    return {"row_loss": (loss, tloss), "lse": (lse, tl), "dX": (dX, tdx), "G": (G, tG),
            "loss": (loss.mean()[None], tloss.mean()[None])}


def _close(got, ref, what):
    value, tol = ref
    off = (got.double() - value).abs()
    worst = (off - tol).max().item()
    assert bool((off <= tol + 1e-30).all()), f"{what}: {worst:.3e} past its tolerance"


SHAPES = [
    (1, 1, 1, 1), (1, 1, 64, 257), (6, 32, 64, 257), (3, 5, 7, 11), (2, 64, 128, 512), (1, 300, 200, 1000),
    (4, 77, 1000, 1031), (5, 1, 40, 300), (1, 257, 72, 255), (2, 130, 520, 2049), (20, 20, 96, 700), (1, 3, 2048, 4000),
]


@pytest.mark.parametrize("x,w", [("bf16", "bf16"), ("f32", "f32"), ("bf16", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("layout", ["dense", "strided", "ragged"])
@pytest.mark.parametrize("N,n_c,C,V", SHAPES)
def test_matches_reference(gc, N, n_c, C, V, x, w, layout):
    X, W, y = _data(N, n_c, C, V, x, w, N + n_c + C + V, layout=layout)
    ref = _reference(X, W, y, N)
    wide = torch.full((N, V * C + 11), -77.0, device="cuda")      # G as a slice of a model's chunk gradients
    first = {"dense": 0, "strided": 8, "ragged": 3}[layout]
    G = wide[:, first:first + V * C]
    dbuf = torch.full((N * n_c, C + 8), -77.0, dtype=X.dtype, device="cuda")
    dX = dbuf[:, first:first + C] if layout != "dense" else True
    ws = gc.Workspace()
    got = gc.gc_softmax_xent(X, W, y if layout != "ragged" else y.int(), N, n_c, G=G, dX=dX, ws=ws)
    gc.gc_status(ws)
    for k in ref:
        _close(got[k], ref[k], k)
    assert (wide[:, :first] == -77).all() and (wide[:, first + V * C:] == -77).all()
    if layout != "dense":
        assert (dbuf[:, :first] == -77).all() and (dbuf[:, first + C:] == -77).all()


@pytest.mark.parametrize("x,w", [("bf16", "bf16"), ("f32", "f32"), ("bf16", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("N,n_c,C,V", [(20, 20, 520, 3000), (3, 700, 600, 9001), (2, 1100, 770, 5000)])
def test_two_pairs_to_a_cluster(gc, N, n_c, C, V, x, w):
    """Enough tiles for clusters of two pairs; the last column tile is half or wholly past the columns."""
    X, W, y = _data(N, n_c, C, V, x, w, N + n_c + C + V)
    ref = _reference(X, W, y, N)
    ws = gc.Workspace()
    got = gc.gc_softmax_xent(X, W, y, N, n_c, ws=ws)
    gc.gc_status(ws)
    for k in ref:
        _close(got[k], ref[k], k)
    again = gc.gc_softmax_xent(X, W, y, N, n_c, ws=ws)
    assert all(torch.equal(got[k], again[k]) for k in got)


@pytest.mark.parametrize("x,w", [("bf16", "bf16"), ("f32", "f32"), ("bf16", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("layout", ["dense", "ragged"])
@pytest.mark.parametrize("T,C,V", [(1, 1, 1), (1, 2048, 5000), (2, 300, 33), (3, 1000, 20001), (4, 64, 12000),
                                   (5, 257, 1000), (8, 520, 4096), (8, 4096, 300), (9, 128, 1000), (1, 16384, 40)])
def test_few_points(gc, T, C, V, x, w, layout):
    """One point takes W as it lies; a few more do not; the same with the gradient asked for."""
    X, W, y = _data(1, T, C, V, x, w, T + C + V, layout=layout)
    ref = _reference(X, W, y, 1)
    ws = gc.Workspace()
    got = gc.gc_softmax_xent(X, W, y, 1, T, dX=False, G=False, ws=ws)
    full = gc.gc_softmax_xent(X, W, y.int(), 1, T, ws=ws)
    gc.gc_status(ws)
    for k in ("loss", "row_loss", "lse"):
        _close(got[k], ref[k], k)
        assert torch.equal(got[k], full[k])
    for k in ("dX", "G"):
        _close(full[k], ref[k], k)


def test_few_points_labels(gc):
    X, W, y = _data(1, 4, 96, 700, "bf16", "bf16", 3, ignore=0)
    want = gc.gc_softmax_xent(X, W, y, 1, 4)
    y2, X2 = y.clone(), X.clone()
    y2[1], y2[3] = -7, 700
    X2[1, 5] = float("nan")
    ws = gc.Workspace()
    got = gc.gc_softmax_xent(X2, W, y2, 1, 4, ws=ws)
    with pytest.raises(gc.GCError) as e:
        gc.gc_status(ws)
    assert e.value.code == -7
    assert torch.equal(got["row_loss"][[0, 2]], want["row_loss"][[0, 2]]) and not got["row_loss"][[1, 3]].any()
    assert torch.equal(got["dX"][[0, 2]], want["dX"][[0, 2]]) and not got["dX"][[1, 3]].any()
    assert torch.isfinite(got["G"]).all() and torch.equal(got["lse"][[0, 2, 3]], want["lse"][[0, 2, 3]])


def test_reference_is_the_oracle(gc):
    X, W, y = _data(3, 6, 10, 40, "f32", "f32", 1)
    ref = _reference(X, W, y, 3)
    loss, lse, dX, G = L.softmax_xent(X.double().cpu(), W.double().cpu(), y.cpu(), 3)
    assert np.allclose(ref["row_loss"][0].cpu(), loss) and np.allclose(ref["dX"][0].cpu(), dX)
    assert np.allclose(ref["G"][0].cpu().view(3, 40, 10), G) and np.allclose(ref["lse"][0].cpu(), lse)


@pytest.mark.parametrize("x,w", [("bf16", "bf16"), ("f32", "f32")])
def test_several_pieces_of_the_vocabulary(gc, x, w):
    """12,000 points: a piece of P holds 2^27 values, so 30,000 columns take three."""
    X, W, y = _data(4, 3000, 72, 30000, x, w, 7)
    ref = _reference(X, W, y, 4)
    ws = gc.Workspace()
    got = gc.gc_softmax_xent(X, W, y, 4, 3000, ws=ws)
    gc.gc_status(ws)
    for k in ref:
        _close(got[k], ref[k], k)


@pytest.mark.parametrize("x", ["bf16", "f32"])
@pytest.mark.parametrize("N,n_c,C,V", [(2, 20, 100, 6000), (1, 300, 136, 20011), (3, 500, 24, 50000), (1, 1, 64, 9000)])
def test_few_tiles_of_the_row_gradient(gc, N, n_c, C, V, x):
    """Few rows and columns against a long vocabulary: the sum over it runs in ranges, added in order."""
    X, W, y = _data(N, n_c, C, V, x, "bf16", N + n_c + C + V, layout="ragged")
    ref = _reference(X, W, y, N)
    ws = gc.Workspace()
    got = gc.gc_softmax_xent(X, W, y, N, n_c, ws=ws)
    gc.gc_status(ws)
    for k in ref:
        _close(got[k], ref[k], k)
    again = gc.gc_softmax_xent(X, W, y, N, n_c, G=False, ws=ws)
    assert torch.equal(again["dX"], got["dX"])


def test_ranges_and_pieces_together(gc):
    """32,000 points and 24 columns: seventeen pieces of 4,096 columns in two ranges each, the last piece of
    one column in one.  Against each half of the points alone (other pieces and ranges): the chunk's
    gradient is the same sum; a bf16 dX rounds another order of it."""
    X, W, y = _data(2, 16000, 24, 16 * 4096 + 1, "bf16", "bf16", 21)
    ws = gc.Workspace()
    got = gc.gc_softmax_xent(X, W, y, 2, 16000, ws=ws)
    gc.gc_status(ws)
    for i in range(2):
        rows = slice(16000 * i, 16000 * i + 16000)
        one = gc.gc_softmax_xent(X[rows], W, y[rows], 1, 16000)
        assert torch.equal(got["G"][i], one["G"][0]) and torch.equal(got["row_loss"][rows], one["row_loss"])
        off = (got["dX"][rows].double() - one["dX"].double()).abs()
        assert (off <= 2 * 2.0 ** -8 * one["dX"].double().abs() + 1e-4).all()


@pytest.mark.parametrize("x,N,n_c,C,V", [("f32", 1, 5569, 384, 4112), ("bf16", 1, 8000, 200, 3000), ("bf16", 2, 1024, 512, 2000),
                                         ("f32", 1, 2000, 64, 30000)])
def test_long_sums_keep_their_digits(gc, x, N, n_c, C, V):
    """32-bit results of sums over thousands of points or columns, in the 2-norm.  Tensor memory is
    added to at most 96 times in a row, each addition cut off by 2^-24 on average, of a running sum
    two thirds of the last: 3.8e-6; the operands' parts are off by 2^-17 at most, 2e-6 on average; z is
    off as the sums are, which moves the probabilities, a smaller part of the results: 8e-6 together."""
    X, W, y = _data(N, n_c, C, V, x, x, n_c + V)
    ref = _reference(X, W, y, N)
    got = gc.gc_softmax_xent(X, W, y, N, n_c)
    for k in ("G", "dX") if x == "f32" else ("G",):
        value = ref[k][0]
        assert ((got[k].double() - value).norm() / value.norm()).item() <= 8e-6, k


def test_outputs_alone_and_repeated(gc):
    X, W, y = _data(3, 200, 136, 900, "bf16", "bf16", 3)
    ws = gc.Workspace()
    full = gc.gc_softmax_xent(X, W, y, 3, 200, ws=ws)
    again = gc.gc_softmax_xent(X, W, y, 3, 200, ws=ws)
    assert all(torch.equal(full[k], again[k]) for k in full)
    only = gc.gc_softmax_xent(X, W, y, 3, 200, dX=False, G=False, ws=ws)
    assert only["dX"] is None and all(torch.equal(only[k], full[k]) for k in ("loss", "row_loss", "lse"))
    assert torch.equal(gc.gc_softmax_xent(X, W, y, 3, 200, G=False, loss=False, row_loss=False, ws=ws)["dX"], full["dX"])
    assert torch.equal(gc.gc_softmax_xent(X, W, y, 3, 200, dX=False, lse=False, ws=ws)["G"], full["G"])
    one = gc.gc_softmax_xent(X, W, y, 3, 200, row_loss=False, lse=False, dX=False, G=False, ws=ws)
    assert torch.equal(one["loss"], full["loss"])


def test_a_chunk_alone_gives_the_same_bits(gc):
    """A worker that holds one chunk sends what any other sends for it."""
    for x in ("bf16", "f32"):
        X, W, y = _data(4, 150, 200, 777, x, "bf16", 13)
        full = gc.gc_softmax_xent(X, W, y, 4, 150)
        one = gc.gc_softmax_xent(X[300:450], W, y[300:450], 1, 150)
        assert torch.equal(one["G"][0], full["G"][2]) and torch.equal(one["dX"], full["dX"][300:450])


def test_rows_without_a_label(gc):
    """Whatever such a row holds, nothing of it is seen; a chunk of them has a zero gradient."""
    X, W, y = _data(3, 50, 100, 300, "bf16", "bf16", 5)
    y[50:100] = -1
    want = gc.gc_softmax_xent(X, W, y, 3, 50)
    bad = X.clone()
    bad[y < 0] = float("nan")
    bad[60] = float("inf")
    got = gc.gc_softmax_xent(bad, W, y, 3, 50)
    assert all(torch.equal(got[k], want[k]) for k in want if k != "lse")
    assert torch.equal(got["lse"][y >= 0], want["lse"][y >= 0]) and got["lse"][y < 0].isnan().all()
    assert torch.isfinite(want["lse"]).all()
    assert not got["G"][1].any() and not got["row_loss"][y < 0].any() and not got["dX"][y < 0].any()
    none = gc.gc_softmax_xent(bad, W, torch.full_like(y, -100), 3, 50)
    assert not none["G"].any() and none["loss"].item() == 0


def test_label_past_the_vocabulary_is_reported(gc):
    X, W, y = _data(1, 40, 64, 300, "bf16", "bf16", 6, ignore=0)
    ws = gc.Workspace()
    y2 = y.clone()
    y2[7] = 300
    got = gc.gc_softmax_xent(X, W, y2, 1, 40, ws=ws)
    with pytest.raises(gc.GCError) as e:
        gc.gc_status(ws)
    assert e.value.code == -7 and "label" in str(e.value)
    gc.gc_status(ws)          # read and cleared
    y2[7] = -1
    want = gc.gc_softmax_xent(X, W, y2, 1, 40, ws=ws)
    assert all(torch.equal(got[k], want[k]) for k in want)


@pytest.mark.parametrize("x", ["bf16", "f32"])
def test_rows_without_a_label_at_the_end_of_the_range(gc, x):
    """The largest fp32 values round to infinity in bf16: in a row without a label they leave no trace."""
    X, W, y = _data(2, 20, 64, 200, x, "bf16", 33, ignore=0)
    y[3] = -1
    want = gc.gc_softmax_xent(X, W, y, 2, 20)
    X[3] = 3.4e38 if x == "f32" else float("inf")
    got = gc.gc_softmax_xent(X, W, y, 2, 20)
    live = y >= 0
    assert torch.equal(got["G"], want["G"]) and torch.equal(got["dX"], want["dX"])
    assert torch.equal(got["lse"][live], want["lse"][live])


@pytest.mark.parametrize("x", ["bf16", "f32"])
def test_losses_alone_of_labels_that_are_none(gc, x):
    """Losses alone take the labels and bf16 rows as they lie: negative labels, labels past the vocabulary
    and rows without a label that are not finite give what they give with the gradient."""
    X, W, y = _data(1, 300, 96, 700, x, "bf16", 31, ignore=0.2)
    y[5], y[6], y[7] = 700, -1, -(1 << 40)
    X[6, 3], X[7, 1] = float("nan"), float("-inf")
    ws = gc.Workspace()
    for labels in (y, y.clamp_min(-(1 << 30)).int()):
        full = gc.gc_softmax_xent(X, W, labels, 1, 300, ws=ws)
        with pytest.raises(gc.GCError) as e:
            gc.gc_status(ws)
        assert e.value.code == -7
        only = gc.gc_softmax_xent(X, W, labels, 1, 300, dX=False, G=False, ws=ws)
        with pytest.raises(gc.GCError):
            gc.gc_status(ws)
        assert torch.equal(only["row_loss"], full["row_loss"]) and torch.equal(only["loss"], full["loss"])
        finite = torch.isfinite(full["lse"])
        assert finite.sum().item() == 298 and torch.equal(only["lse"][finite], full["lse"][finite])
        assert not torch.isfinite(only["lse"][~finite]).any()


def test_nonfinite_rows_stay_in_their_chunk(gc):
    X, W, y = _data(3, 40, 64, 500, "bf16", "bf16", 8, ignore=0)
    want = gc.gc_softmax_xent(X, W, y, 3, 40)
    X[45, 3] = float("inf")
    got = gc.gc_softmax_xent(X, W, y, 3, 40)
    assert not torch.isfinite(got["row_loss"][45]) and not torch.isfinite(got["G"][1]).all()
    for i in (0, 2):
        rows = slice(40 * i, 40 * i + 40)
        assert torch.equal(got["G"][i], want["G"][i]) and torch.equal(got["dX"][rows], want["dX"][rows])
        assert torch.equal(got["row_loss"][rows], want["row_loss"][rows])


def test_large_logits(gc):
    """Logits of spread 60 (probabilities of 0 and 1): no overflow, the same tolerances."""
    X, W, y = _data(2, 100, 128, 600, "bf16", "bf16", 9, scale=60.0)
    ref = _reference(X, W, y, 2)
    got = gc.gc_softmax_xent(X, W, y, 2, 100)
    for k in ref:
        _close(got[k], ref[k], k)


def test_gradients_against_differences_of_the_loss(gc):
    """Central differences of the GPU's own summed loss along a direction.  A loss of about 7 is off by
    about 2^-20 7; 60 of them over 2 t, t = 2^-6: below 1e-2; the cubic term is t^2 = 2.4e-4 of a
    derivative of order 100: 3e-2 in all, doubled."""
    N, n_c, C, V = 2, 30, 50, 400
    X, W, y = _data(N, n_c, C, V, "f32", "f32", 10)
    g = torch.Generator(device="cuda").manual_seed(11)
    s, q = torch.randn(N * n_c, C, generator=g, device="cuda"), torch.randn(V, C, generator=g, device="cuda") / C ** 0.5
    out = gc.gc_softmax_xent(X, W, y, N, n_c)
    total = lambda a, b: gc.gc_softmax_xent(a, b, y, N, n_c, dX=False, G=False)["row_loss"].double()
    t = 2.0 ** -6
    dx = (total(X + t * s, W) - total(X - t * s, W)).sum().item() / (2 * t)
    assert abs(dx - (out["dX"].double() * s).sum().item()) <= 6e-2
    dw = (total(X, W + t * q) - total(X, W - t * q)).view(N, n_c).sum(1) / (2 * t)
    want = (out["G"].view(N, V, C).double() * q).sum((1, 2))
    assert (dw - want).abs().max().item() <= 6e-2


def test_on_another_stream_and_in_a_graph(gc):
    X, W, y = _data(2, 64, 128, 700, "bf16", "bf16", 12)
    want = gc.gc_softmax_xent(X * 2, W, y, 2, 64)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    ws = gc.Workspace()
    out = {"G": torch.empty(2, 700 * 128, device="cuda"), "dX": torch.empty_like(X)}
    with torch.cuda.stream(s):
        got = gc.gc_softmax_xent(X * 2, W, y, 2, 64, ws=ws, **out)
    s.synchronize()
    assert all(torch.equal(got[k], want[k]) for k in want)
    X2 = X * 2
    out["G"].zero_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        gc.gc_softmax_xent(X2, W, y, 2, 64, ws=ws, loss=False, row_loss=False, lse=False, **out)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out["G"], want["G"]) and torch.equal(out["dX"], want["dX"])


def test_stall_times_out_then_recovers(gc):
    """The failure path without a fault: the loads are withheld, the waits expire, the status says so
    and the next call is right."""
    X, W, y = _data(2, 300, 256, 1500, "bf16", "bf16", 14)
    want = gc.gc_softmax_xent(X, W, y, 2, 300)
    ws = gc.Workspace()
    gc.gc_set_wait_limit(1 << 22)
    try:
        gc.gc_inject_stall(gc.GC_STALL_XENT)
        gc.gc_softmax_xent(X, W, y, 2, 300, dX=False, G=False, ws=ws)
        torch.cuda.synchronize()
        with pytest.raises(gc.GCError) as e:
            gc.gc_status(ws)
        assert e.value.code == -5
    finally:
        gc.gc_inject_stall(0)
        gc.gc_set_wait_limit(0)
    got = gc.gc_softmax_xent(X, W, y, 2, 300, ws=ws)
    gc.gc_status(ws)
    assert all(torch.equal(got[k], want[k]) for k in want)


@pytest.mark.parametrize("T,C", [(1, 40), (40, 96), (300, 257)])
def test_row_gradient_keeps_the_digits_of_fp32_weights(gc, T, C):
    """Two classes of equal logits: P is 1/2 and -1/2 and dX half the difference of W's rows, 1 + at most
    2^-7 each, which W's first bf16 part alone does not hold.  Both parts are off by 2^-17 a row, P is off by
    2^-20, two additions in tensor memory by 2^-23: 2^-15 together, beside dX's own rounding."""
    g = torch.Generator(device="cuda").manual_seed(T + C)
    W = 1 + (torch.rand(2, C, generator=g, device="cuda") - 0.5) * 2.0 ** -6
    W[:, 0] = 0
    X = torch.zeros(T, C, dtype=torch.bfloat16, device="cuda")
    X[:, 0] = torch.randn(T, generator=g, device="cuda").bfloat16()
    y = torch.randint(0, 2, (T,), generator=g, device="cuda")
    want = 0.5 * (W[1 - y].double() - W[y].double())
    got = gc.gc_softmax_xent(X, W, y, 1, T)["dX"].double()
    assert ((got - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -15).all()


@pytest.mark.parametrize("x", ["bf16", "f32"])
@pytest.mark.parametrize("N,n_c,C,V", [(8, 1024, 64, 20000), (24, 256, 40, 9000)])
def test_a_chunk_alone_gives_the_same_bits_beside_many(gc, N, n_c, C, V, x):
    """The sums of the losses are joined in one order, however many points the call has."""
    X, W, y = _data(N, n_c, C, V, x, "bf16", N + V)
    full = gc.gc_softmax_xent(X, W, y, N, n_c)
    rows = slice(2 * n_c, 3 * n_c)
    one = gc.gc_softmax_xent(X[rows], W, y[rows], 1, n_c)
    assert torch.equal(one["lse"], full["lse"][rows]) and torch.equal(one["row_loss"], full["row_loss"][rows])
    assert torch.equal(one["G"][0], full["G"][2])


@pytest.mark.parametrize("x,w", [("bf16", "bf16"), ("f32", "f32"), ("bf16", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("layout", ["dense", "ragged"])
def test_a_chunk_of_one_point_alone_gives_the_same_bits(gc, x, w, layout):
    X, W, y = _data(5, 1, 200, 3001, x, w, 17, ignore=0, layout=layout)
    full = gc.gc_softmax_xent(X, W, y, 5, 1)
    for i in range(5):
        one = gc.gc_softmax_xent(X[i:i + 1], W, y[i:i + 1], 1, 1)
        assert torch.equal(one["G"][0], full["G"][i])


@pytest.mark.parametrize("x", ["bf16", "f32"])
@pytest.mark.parametrize("label", [-1, 7])
def test_rows_at_the_end_of_the_range_are_finite(gc, x, label):
    """The largest values of X's type are values: the row's logits are finite (W is small there), and so is
    what comes of them, with a label or without, with the gradient or without it."""
    X, W, y = _data(2, 20, 64, 200, x, "f32", 41, ignore=0)
    X[3, 5], W[:, 5] = torch.finfo(X.dtype).max, 2.0 ** -122
    W[9, 5] = 2.0 ** -121
    y[3] = label
    z = X.double() @ W.double().T
    lse = torch.logsumexp(z, 1)
    tz = (20 * 2.0 ** -23 + 2.0 ** -15) * (X.double().abs() @ W.double().abs().T)
    tol = tz.amax(1) + 2.0 ** -20 * (1 + lse + z.abs().amax(1))
    full, only = gc.gc_softmax_xent(X, W, y, 2, 20), gc.gc_softmax_xent(X, W, y, 2, 20, dX=False, G=False)
    for got in (full, only):
        assert ((got["lse"].double() - lse).abs() <= tol).all()
        assert torch.isfinite(got["row_loss"]).all()
    assert torch.equal(full["lse"], only["lse"]) and torch.equal(full["row_loss"], only["row_loss"])
    assert torch.isfinite(full["dX"]).all()
    if label < 0:
        want = gc.gc_softmax_xent(torch.where(y[:, None] < 0, torch.zeros_like(X), X), W, y, 2, 20)
        assert torch.equal(full["G"], want["G"]) and torch.equal(full["dX"], want["dX"])


@pytest.mark.parametrize("x,w,C", [("bf16", "bf16", 32768), ("f32", "f32", 16384), ("bf16", "f32", 16384), ("bf16", "bf16", 4160)])
def test_logits_of_long_rows_keep_their_digits(gc, x, w, C):
    """Products of one sign, whose sum loses most where additions cut off.  At most 128 of them, and 16 products
    each, are added in tensor memory in a row, each off by at most 2^-23 of the sum; the sums of those are
    rounded (2^-24 each); operands in two parts are off by 2^-15 together.  lse adds 2^-20."""
    T, V = 40, 300
    g = torch.Generator(device="cuda").manual_seed(C)
    X = torch.rand(T, C, generator=g, device="cuda").add_(0.5).to(TYPES[x])
    W = torch.rand(V, C, generator=g, device="cuda").add_(0.5).mul_(30.0 / C).to(TYPES[w])
    y = torch.randint(0, V, (T,), generator=g, device="cuda")
    z = X.double() @ W.double().T
    lse = torch.logsumexp(z, 1)
    parts = 2.0 ** -15 if "f32" in (x, w) else 0.0
    top = z.amax(1)
    tz = (144 * 2.0 ** -23 + (C / 640 + 1) * 2.0 ** -24 + parts) * top
    tl = tz + 2.0 ** -20 * (1 + lse.abs() + top)
    loss = lse - z.gather(1, y[:, None])[:, 0]
    ws = gc.Workspace()
    for grad in (False, True):
        got = gc.gc_softmax_xent(X, W, y, 1, T, dX=grad, G=grad, ws=ws)
        gc.gc_status(ws)
        assert ((got["lse"].double() - lse).abs() <= tl).all()
        assert ((got["row_loss"].double() - loss).abs() <= tl + tz).all()
    # the columns of P add to nothing in every row, as far as P and lse come from the same z
    P = torch.softmax(z, 1).scatter_add(1, y[:, None], torch.full((T, 1), -1.0, dtype=torch.float64, device="cuda"))
    tp = P.abs() * (tz + tl)[:, None] + 2.0 ** -16 * P.abs()
    G = got["G"].view(V, C).double()
    assert ((G - P.T @ X.double()).abs() <= (tp.T @ X.double()) + 2.0 ** -15 * (P.abs().T @ X.double())).all()
