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
