"""ctypes binding of libgc.so (argument marshalling only).

Tensors passed to device entry points must be contiguous CUDA tensors of the
dtype the C header states; outputs not supplied by the caller are allocated
with torch.  Calls are asynchronous on torch's current stream, like the C
functions; gc_status() synchronises and reports device-detected data errors.
"""
from __future__ import annotations

import ctypes
import functools
import os

import numpy as np
import torch  # loads the CUDA runtime libgc.so links against

_HERE = os.path.dirname(os.path.abspath(__file__))
library_path = os.path.join(_HERE, "libgc.so")
if not os.path.exists(library_path):
    raise ImportError(
        f"{library_path} is missing: build it with `python -c 'import __graft_entry__ as g; g.build()'`"
        " (the gradient-coding path has no fallback without the CUDA library)")
lib = ctypes.CDLL(library_path)

GC_CYCLIC, GC_EXPLICIT = 0, 1
GC_F32, GC_BF16 = 0, 1
GC_LSQ, GC_LOGISTIC = 0, 1
GC_ACT_NONE, GC_ACT_RELU, GC_ACT_GELU, GC_ACT_GELU_TANH, GC_ACT_SILU = range(5)

_i, _sz, _p, _d, _f, _i64, _u64 = (ctypes.c_int, ctypes.c_size_t, ctypes.c_void_p, ctypes.c_double,
                                   ctypes.c_float, ctypes.c_int64, ctypes.c_uint64)


def _sig(name, res, *args):
    fn = getattr(lib, name)
    fn.restype = res
    fn.argtypes = list(args)
    return fn


_sig("gc_last_error", ctypes.c_char_p)
_sig("gc_version", _i)
_sig("gc_kernel_launches", ctypes.c_uint64)
_sig("gc_set_wait_limit", _i, _i64)
_sig("gc_inject_stall", _i, _i)
_sig("gc_set_decode_policy", _i, _i)
_sig("gc_workspace_init", _i, _p, _sz, _p)
_sig("gc_status", _i, _p, _p)
_sig("gc_make_assignment", _i, _i, _i, _i, _i, _p, _p, _p, _p)
_sig("gc_chunk_ordering", _i, _p, _i, _i, _i, _p, _p)
_sig("gc_trigger_workspace", _sz, _i)
_sig("gc_chunk_grads_batched_workspace", _sz, _i, _i, _i, _i)
_sig("gc_chunk_grads_batched", _i, _p, _p, _p, _i, _i, _i, _i, _i, _p, _p, _sz, _p)
_sig("gc_trigger_times", _i, _p, _i, _i, _i, _p, _i64, _i, _i, _p, _p, _p, _p, _sz, _p)
_sig("gc_chunk_grads_workspace", _sz, _i, _i, _i, _i)
_sig("gc_chunk_grads", _i, _p, _i, _p, _p, _i, _i, _i, _i, _p, _p, _p, _sz, _p)
_sig("gc_coeff_workspace", _sz, _i, _i, _i, _i, _i)
_sig("gc_find_encoding_coeff", _i, _p, _i, _p, _i, _i, _i, _p, _i, _p, _p, _p, _p, _p, _p, _p,
     _sz, _p)
_sig("gc_find_encoding_coeff_noalloc", _i, _p, _i, _p, _i, _i, _i, _p, _i, _p, _p, _p, _p, _p, _p,
     _p)
_sig("gc_encode_workspace", _sz, _i, _i, _i, _i, _i, _i)
_sig("gc_encode", _i, _p, _i, _p, _i, _i, _i, _p, _i, _p, _i, _p, _p, _sz, _p)
_sig("gc_encode_with_coeffs", _i, _p, _i, _p, _i, _i, _i, _p, _i, _p, _i, _p, _p)
_sig("gc_decode_tx", _i, _p, _i, _i, _p, _i, _i, _p, _p)
_sig("gc_decode_batch_workspace", _sz, _i, _i, _i, _i, _i, _i)
_sig("gc_decode_batch", _i, _p, _i, _p, _i, _i, _i, _p, _i, _p, _i, _p, _p, _p, _p, _p, _sz, _p)
_sig("gc_decode_plan_bytes", _sz, _i, _i, _i)
_sig("gc_decode_plan_workspace", _sz, _i, _i, _i, _i, _i)
_sig("gc_decode_plan", _i, _p, _i, _p, _i, _i, _i, _p, _i, _p, _sz, _p, _p, _p, _sz, _p)
_sig("gc_decode_prepare_bytes", _sz, _i, _i, _i, _i)
_sig("gc_decode_prepare", _i, _p, _i, _p, _i, _i, _i, _p, _sz, _p)
_sig("gc_decode_plan_prepared_workspace", _sz)
_sig("gc_decode_plan_prepared", _i, _p, _p, _i, _i, _i, _i, _p, _i, _p, _sz, _p, _p, _p, _sz, _p)
_sig("gc_decode_apply_workspace", _sz, _i, _i, _i, _i)
_sig("gc_decode_apply", _i, _p, _i, _i, _i, _p, _i, _p, _p, _p, _sz, _p)
_sig("gc_decode_combine_workspace", _sz, _i, _i, _i, _i)
_sig("gc_decode_combine", _i, _p, _i, _i, _i, _p, _i, _p, _p, _p, _sz, _p)
_sig("gc_mse_workspace", _sz, _i, _i, _i, _i, _i, _i)
_sig("gc_mse", _i, _p, _i, _p, _i, _i, _i, _p, _i, _p, _i, _p, _p, _p, _p, _sz, _p)
_sig("gc_sgd_step", _i, _p, _p, _i, _f, _i64, _p)
_sig("gc_live_step", _i, _p, _p, _i, _p, _i, _i, _i, _p, _p, _i, _f, _i64, _p, _p, _p, _p)
_sig("gc_dropout", _i, _p, _i64, _p, _i64, _i, _i64, _i, _d, _u64, _u64, _i64, _p, _i64, _p)
_sig("gc_layer_norm", _i, _p, _i64, _p, _i64, _i, _i64, _i, _p, _p, _f, _d, _u64, _u64, _i64, _p, _i64,
     _p, _i64, _p, _p, _p)
_sig("gc_layer_norm_backward_workspace", _sz, _i, _i, _i)
_sig("gc_layer_norm_backward", _i, _p, _i64, _p, _i64, _p, _p, _p, _p, _i64, _i, _i, _i, _i, _d, _u64,
     _u64, _i64, _p, _i64, _p, _i64, _p, _i64, _p, _sz, _p)
_sig("gc_softmax_xent_workspace", _sz, _i, _i, _i, _i, _i, _i, _i, _i)
_sig("gc_softmax_xent", _i, _p, _i64, _i, _p, _i64, _i, _p, _i, _i, _i, _i, _i, _p, _p, _p, _p, _i64, _p,
     _i64, _p, _sz, _p)

_sig("gc_linear_workspace", _sz, _i64, _i, _i, _i, _i, _i, _i)
_sig("gc_linear", _i, _p, _i64, _i, _p, _i64, _i, _p, _i, _p, _i64, _i64, _i, _i, _p, _i64, _p, _i64, _p, _sz,
     _p)
_sig("gc_linear_backward_workspace", _sz, *[_i] * 11)
_sig("gc_linear_backward", _i, _p, _i64, _p, _i64, _p, _i64, _i, _p, _i64, _i, _i, _i, _i, _i, _i, _p, _i64, _p,
     _i64, _p, _i64, _p, _sz, _p)

_sig("gc_orthogonalize_workspace", _sz, _i, _i, _i, _i)
_sig("gc_orthogonalize", _i, _p, _i64, _i64, _i, _i, _i, _i, _p, _i, _f, _p, _i64, _i64, _p, _sz, _p)
_sig("gc_muon_step", _i, _p, _i64, _i64, _p, _i64, _i64, _p, _i64, _i64, _i, _i, _i, _f, _i64, _f, _i, _f, _f, _p, _i,
     _f, _p, _sz, _p)


class GCError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"gc error {code}: {msg}")
        self.code = code


def gc_last_error() -> str:
    return lib.gc_last_error().decode()


def gc_version() -> int:
    return lib.gc_version()


def _check(rc: int) -> None:
    if rc != 0:
        raise GCError(rc, gc_last_error())


def block_length(d: int, ell: int) -> int:
    return -(-d // ell)


# The raw handle of torch's current stream (building a Stream object for it costs 2 us a call).
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(device=None) -> int:
    if _raw_stream is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(torch.cuda.current_device() if device is None else device)


@functools.lru_cache(maxsize=1024)
def _bytes(query, *sizes) -> int:
    """A workspace size, a function of the sizes alone, asked of the library once."""
    return int(getattr(lib, query)(*sizes))


@functools.lru_cache(maxsize=1024)
def _device_bytes(device, query, *sizes) -> int:
    """... of the sizes and of the number of SMs of the current device."""
    return int(getattr(lib, query)(*sizes))


def _dev(t, dtype, name, shape=None):
    """Device pointer of a contiguous CUDA tensor of the given dtype (None -> NULL)."""
    if t is None:
        return None
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA tensor")
    if t.dtype is not dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if shape is not None and t.shape != shape:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    return t.data_ptr()


def _rows(t, dtype, name, shape):
    """(device pointer, row stride) of a CUDA matrix whose rows may lie apart (None -> NULL, 0)."""
    if t is None:
        return None, 0
    if isinstance(t, torch.Tensor) and t.is_cuda and t.dtype is dtype and t.shape == shape:
        ld, one = t.stride()
        if (one == 1 or shape[1] <= 1) and (ld >= shape[1] or shape[0] <= 1):
            return t.data_ptr(), ld
        raise ValueError(f"the rows of {name} overlap" if one == 1 or shape[1] <= 1 else
                         f"the elements of a row of {name} must lie next to each other")
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA tensor")
    if t.dtype is not dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")


def _elt(t, name):
    if not isinstance(t, torch.Tensor) or t.dim() != 2:
        raise TypeError(f"{name} must be a matrix")
    if t.dtype is torch.bfloat16:
        return GC_BF16
    if t.dtype is torch.float32:
        return GC_F32
    raise TypeError(f"{name} must be float32 or bfloat16")


class Workspace:
    """Reusable device scratch buffer; grows on demand.  Its 256-byte status
    header is zeroed whenever a new buffer is allocated."""

    def __init__(self, device=None):
        self.device = torch.device(device) if device is not None else torch.device("cuda")
        self.buf = None

    def get(self, nbytes: int):
        nbytes = max(int(nbytes), 256)
        if self.buf is None or self.buf.numel() < nbytes:
            self.buf = None
            self.buf = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
            _check(lib.gc_workspace_init(self.buf.data_ptr(), nbytes, _stream()))
        return self.buf.data_ptr(), self.buf.numel()

    def status(self) -> None:
        if self.buf is not None:
            _check(lib.gc_status(self.buf.data_ptr(), _stream()))


def _ws(ws, nbytes, device):
    if ws is None:
        ws = Workspace(device)
    return ws, ws.get(nbytes)


def gc_status(ws: Workspace) -> None:
    """Synchronise and raise GCError if a kernel flagged bad data or a timeout."""
    ws.status()


# ---------------------------------------------------------------- assignment
def gc_make_assignment(N: int, m: int, delta: int, kind: int = GC_CYCLIC, explicit_order=None):
    """Host-only: (A N x m uint8, order m x delta int32, O N x m uint8) numpy arrays."""
    A = np.zeros((N, m), dtype=np.uint8)
    O = np.zeros((N, m), dtype=np.uint8)
    order = np.zeros((m, delta), dtype=np.int32)
    ex = None
    if explicit_order is not None:
        ex = np.ascontiguousarray(explicit_order, dtype=np.int32)
        if ex.shape != (m, delta):
            raise ValueError("explicit_order must be m x delta")
    _check(lib.gc_make_assignment(N, m, delta, kind, None if ex is None else ex.ctypes.data,
                                  A.ctypes.data, order.ctypes.data, O.ctypes.data))
    return A, order, O


def gc_chunk_ordering(A):
    """Host-only Algorithm 2: A (N x N, every row and column sum delta) ->
    (order m x delta int32, O N x m uint8) with every row sum of O equal to
    delta (delta + 1) / 2."""
    A = np.ascontiguousarray(np.asarray(A) != 0, dtype=np.uint8)
    N, m = A.shape
    delta = int(A[0].sum()) if N else 0
    order = np.zeros((m, max(delta, 1)), dtype=np.int32)
    O = np.zeros((N, m), dtype=np.uint8)
    _check(lib.gc_chunk_ordering(A.ctypes.data, N, m, delta, order.ctypes.data, O.ctypes.data))
    return order, O


def gc_trigger_times(order, N: int, m: int, delta: int, tau, ell: int, theta: int = 0, T=True,
                     psi=True, T_full=True, ws: Workspace | None = None):
    """Completion times and the encode-and-transmit trigger for nsim simulated
    realizations (tau: nsim x m float64 on the device, +inf = failed worker).
    Returns dict T (nsim float64), psi (nsim x m int32), T_full (nsim float64);
    pass a tensor to write into it or False to skip an output."""
    nsim = tau.shape[0]
    dev = tau.device

    def out(x, shape, dt):
        if x is True:
            return torch.empty(shape, dtype=dt, device=dev)
        return x if isinstance(x, torch.Tensor) else None
    T = out(T, (nsim,), torch.float64)
    psi = out(psi, (nsim, m), torch.int32)
    T_full = out(T_full, (nsim,), torch.float64)
    ws, (wp, wn) = _ws(ws, _bytes("gc_trigger_workspace", N), dev)
    _check(lib.gc_trigger_times(
        _dev(order, torch.int32, "order", (m, delta)), N, m, delta,
        _dev(tau, torch.float64, "tau", (nsim, m)), nsim, ell, theta,
        _dev(T, torch.float64, "T", (nsim,)), _dev(psi, torch.int32, "psi", (nsim, m)),
        _dev(T_full, torch.float64, "T_full", (nsim,)), wp, wn, _stream()))
    return {"T": T, "psi": psi, "T_full": T_full}


def gc_chunk_grads_batched(X, y, W, N: int, n_c: int, loss: int, G=None,
                           ws: Workspace | None = None):
    """Chunk gradients for n_w parameter vectors (rows of W) on the tensor
    cores: G (n_w x N x d float32).  X must be bfloat16."""
    n_w, d = W.shape
    if X.dtype != torch.bfloat16:
        raise TypeError("X must be bfloat16")
    if G is None:
        G = torch.empty(n_w, N, d, dtype=torch.float32, device=X.device)
    ws, (wp, wn) = _ws(ws, _device_bytes(torch.cuda.current_device(), "gc_chunk_grads_batched_workspace",
                                        N, n_c, d, n_w), X.device)
    _check(lib.gc_chunk_grads_batched(
        _dev(X, torch.bfloat16, "X", (N * n_c, d)), _dev(y, torch.float32, "y", (N * n_c,)),
        _dev(W, torch.float32, "W", (n_w, d)), N, n_c, d, n_w, loss,
        _dev(G, torch.float32, "G", (n_w, N, d)), wp, wn, _stream()))
    return G


# ---------------------------------------------------------------- chunk gradients
def gc_chunk_grads_workspace(N, n_c, d, x_dtype):
    return lib.gc_chunk_grads_workspace(N, n_c, d, x_dtype)


def gc_chunk_grads(X, y, w, N: int, n_c: int, loss: int, G=None, loss_out=None,
                   ws: Workspace | None = None):
    """G (N x d float32) = per-chunk gradients; loss_out (1 float64) optional."""
    d = X.shape[1]
    x_dtype = GC_BF16 if X.dtype == torch.bfloat16 else GC_F32
    if X.dtype not in (torch.float32, torch.bfloat16):
        raise TypeError("X must be float32 or bfloat16")
    if X.shape[0] != N * n_c:
        raise ValueError("X must have N * n_c rows")
    if G is None:
        G = torch.empty(N, d, dtype=torch.float32, device=X.device)
    ws, (wp, wn) = _ws(ws, _device_bytes(torch.cuda.current_device(), "gc_chunk_grads_workspace",
                                        N, n_c, d, x_dtype), X.device)
    _check(lib.gc_chunk_grads(_dev(X, X.dtype, "X"), x_dtype, _dev(y, torch.float32, "y", (N * n_c,)),
                              _dev(w, torch.float32, "w", (d,)), N, n_c, d, loss,
                              _dev(G, torch.float32, "G", (N, d)),
                              _dev(loss_out, torch.float64, "loss_out"), wp, wn, _stream()))
    return G


# ---------------------------------------------------------------- dropout, layer norm
def gc_dropout(x, p: float, seed: int, offset: int = 0, row0: int = 0, residual=None, out=None):
    """residual + D(x) (rows x cols): D drops an element with probability p and scales the others, by
    a mask that is a function of (seed, offset, row0 + row, column) and is never stored.  The
    gradient of D is gc_dropout of the gradient with the same numbers.  Rows may be strided."""
    dt = _elt(x, "x")
    if out is None:
        out = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    xp, ldx = _rows(x, x.dtype, "x", x.shape)
    rp, ldr = _rows(residual, x.dtype, "residual", x.shape)
    op, ldo = _rows(out, x.dtype, "out", x.shape)
    _check(lib.gc_dropout(xp, ldx, rp, ldr, dt, x.shape[0], x.shape[1], p, seed, offset, row0, op, ldo,
                          _stream()))
    return out


def gc_layer_norm(x, gamma=None, beta=None, eps: float = 1e-5, residual=None, p: float = 0.0,
                  seed: int = 0, offset: int = 0, row0: int = 0, y=None, h=None, mean=True, rstd=True):
    """y = layer norm of h = residual + D(x) (gc_dropout's D; h = x without both).  Returns dict with
    y, h (x itself where there is neither residual nor dropout, no tensor is given for it and y is not
    written over x), and mean, rstd (rows, float32; None where False is passed): what
    gc_layer_norm_backward takes."""
    dt = _elt(x, "x")
    rows, cols = x.shape
    dev = x.device
    over = isinstance(y, torch.Tensor) and y.data_ptr() == x.data_ptr()
    if y is None:
        y = torch.empty(x.shape, dtype=x.dtype, device=dev)
    if h is None and (residual is not None or p > 0 or over):
        h = torch.empty(x.shape, dtype=x.dtype, device=dev)
    if mean is True:
        mean = torch.empty(rows, dtype=torch.float32, device=dev)
    if rstd is True:
        rstd = torch.empty(rows, dtype=torch.float32, device=dev)
    if not isinstance(mean, torch.Tensor):
        mean = None
    if not isinstance(rstd, torch.Tensor):
        rstd = None
    xp, ldx = _rows(x, x.dtype, "x", x.shape)
    rp, ldr = _rows(residual, x.dtype, "residual", x.shape)
    yp, ldy = _rows(y, x.dtype, "y", x.shape)
    hp, ldh = _rows(h, x.dtype, "h", x.shape)
    _check(lib.gc_layer_norm(xp, ldx, rp, ldr, dt, rows, cols,
                             _dev(gamma, torch.float32, "gamma", (cols,)),
                             _dev(beta, torch.float32, "beta", (cols,)), eps, p, seed, offset, row0, yp,
                             ldy, hp, ldh, _dev(mean, torch.float32, "mean", (rows,)),
                             _dev(rstd, torch.float32, "rstd", (rows,)), _stream()))
    return {"y": y, "h": x if h is None else h, "mean": mean, "rstd": rstd}


def gc_layer_norm_backward(dy, h, mean, rstd, gamma, N: int, n_c: int, dh=None, p: float = 0.0,
                           seed: int = 0, offset: int = 0, row0: int = 0, dx=True, dresidual=False,
                           G=True, ws: Workspace | None = None):
    """Gradient of gc_layer_norm.  Returns dict with dx (of x), dresidual (of residual) and G (N x 2 cols
    float32: per chunk the sums for gamma, then those for beta); booleans ask for an output, tensors
    are written into (G may be a column slice of a larger matrix of chunk gradients)."""
    dt = _elt(dy, "dy")
    rows, cols = dy.shape
    if rows != N * n_c:
        raise ValueError("dy must have N * n_c rows")
    dev = dy.device

    def out(t, shape, dtype):
        if isinstance(t, torch.Tensor):
            return t
        return torch.empty(shape, dtype=dtype, device=dev) if t else None
    dx, dresidual = out(dx, dy.shape, dy.dtype), out(dresidual, dy.shape, dy.dtype)
    G = out(G, (N, 2 * cols), torch.float32)
    yp, lddy = _rows(dy, dy.dtype, "dy", dy.shape)
    hp, ldh = _rows(h, dy.dtype, "h", dy.shape)
    ap, lddh = _rows(dh, dy.dtype, "dh", dy.shape)
    xp, lddx = _rows(dx, dy.dtype, "dx", dy.shape)
    rp, lddr = _rows(dresidual, dy.dtype, "dresidual", dy.shape)
    gp, ldg = _rows(G, torch.float32, "G", (N, 2 * cols))
    ws, (wp, wn) = _ws(ws, _device_bytes(torch.cuda.current_device(), "gc_layer_norm_backward_workspace",
                                        N, n_c, cols), dev)
    _check(lib.gc_layer_norm_backward(
        yp, lddy, hp, ldh, _dev(mean, torch.float32, "mean", (rows,)),
        _dev(rstd, torch.float32, "rstd", (rows,)), _dev(gamma, torch.float32, "gamma", (cols,)), ap, lddh,
        dt, N, n_c, cols, p, seed, offset, row0, xp, lddx, rp, lddr, gp, ldg, wp, wn, _stream()))
    return {"dx": dx, "dresidual": dresidual, "G": G}


# ---------------------------------------------------------------- softmax cross entropy
def gc_softmax_xent(X, W, y, N: int, n_c: int, loss=True, row_loss=True, lse=True, dX=True, G=True,
                    ws: Workspace | None = None):
    """Softmax cross entropy of the rows X W^T (X N n_c x C, W V x C, float32 or bfloat16 each) at the
    labels y (int64 or int32; negative: none), with its gradient, neither logits nor probabilities
    kept.  Returns dict with loss (1 float64, the mean over all points), row_loss, lse (float32), dX
    (X's type) and G (N x V C float32: per chunk the gradient of W, un-normalised); booleans ask for
    an output, tensors are written into (G may be a column slice of a larger matrix)."""
    xt, wt = _elt(X, "X"), _elt(W, "W")
    T, C = X.shape
    V = W.shape[0]
    if T != N * n_c:
        raise ValueError("X must have N * n_c rows")
    if y.dtype is not torch.int64 and y.dtype is not torch.int32:
        raise TypeError("y must be int64 or int32")
    dev = X.device

    def out(t, shape, dtype):
        if isinstance(t, torch.Tensor):
            return t
        return torch.empty(shape, dtype=dtype, device=dev) if t else None
    loss, row_loss = out(loss, (1,), torch.float64), out(row_loss, (T,), torch.float32)
    lse = out(lse, (T,), torch.float32)
    dX, G = out(dX, X.shape, X.dtype), out(G, (N, V * C), torch.float32)
    xp, ldx = _rows(X, X.dtype, "X", X.shape)
    wp_, ldw = _rows(W, W.dtype, "W", (V, C))
    dp, lddx = _rows(dX, X.dtype, "dX", X.shape)
    gp, ldg = _rows(G, torch.float32, "G", (N, V * C))
    e = W.element_size()
    w_16 = int(wp_ % 16 == 0 and (ldw * e % 16 == 0 or V == 1))
    ws, (wp, wn) = _ws(ws, _device_bytes(torch.cuda.current_device(), "gc_softmax_xent_workspace", N, n_c, C,
                                        V, xt, wt, w_16, (dX is not None) + 2 * (G is not None)), dev)
    _check(lib.gc_softmax_xent(
        xp, ldx, xt, wp_, ldw, wt, _dev(y, y.dtype, "y", (T,)), int(y.dtype is torch.int64), N, n_c, C, V,
        _dev(loss, torch.float64, "loss"), _dev(row_loss, torch.float32, "row_loss", (T,)),
        _dev(lse, torch.float32, "lse", (T,)), dp, lddx, gp, ldg, wp, wn, _stream()))
    return {"loss": loss, "row_loss": row_loss, "lse": lse, "dX": dX, "G": G}


# ---------------------------------------------------------------- linear layers
def _out(t, rows, cols, dtype, device, name):
    """(an output, its device pointer, its row stride): the tensor given, one made for True, None for False."""
    if isinstance(t, torch.Tensor):
        return t, *_rows(t, dtype, name, (rows, cols))
    if not t:
        return None, None, 0
    t = torch.empty((rows, cols), dtype=dtype, device=device)
    return t, t.data_ptr(), cols


def _on_16(ptr, ld, rows, elt):
    """Whether rows lie on 16-byte boundaries (a single one needs no stride)."""
    return 1 if ptr is not None and not (ptr & 15) and (not (ld * elt & 15) or rows == 1) else 0


def _same_device(*tensors):
    """The current device: calls run on its stream, with its tensors alone."""
    here = torch.cuda.current_device()
    for t in tensors:
        if t is not None and t.get_device() != here:
            raise ValueError(f"a tensor on {t.device}, but the current device is cuda:{here}")
    return here


def gc_linear(x, W, bias=None, act: int = GC_ACT_NONE, residual=None, y=None, z=False,
              ws: Workspace | None = None):
    """y = residual + act(z), z = x W^T + bias (x rows x C, W F x C, float32 or bfloat16 each, bias F
    float32).  Returns dict with y (x's type; a tensor given is written into, and may be the residual) and z
    (None unless True or a tensor is given: what gc_linear_backward takes).  Rows may be strided."""
    xt, wt = _elt(x, "x"), _elt(W, "W")
    dt, (rows, C) = x.dtype, x.shape
    F = W.shape[0]
    xp, ldx = _rows(x, dt, "x", (rows, C))
    wp_, ldw = _rows(W, W.dtype, "W", (F, C))
    rp, ldr = _rows(residual, dt, "residual", (rows, F))
    bp = _dev(bias, torch.float32, "bias", (F,))
    y, yp, ldy = _out(True if y is None else y, rows, F, dt, x.device, "y")
    z, zp, ldz = _out(z, rows, F, dt, x.device, "z")
    here = _same_device(x, W, bias, residual, y, z)
    ws, (wp, wn) = _ws(ws, _device_bytes(here, "gc_linear_workspace", rows, C, F, xt, wt, _on_16(xp, ldx, rows, 4 - 2 * xt),
                                        _on_16(wp_, ldw, F, 4 - 2 * wt)), x.device)
    _check(lib.gc_linear(xp, ldx, xt, wp_, ldw, wt, bp, act, rp, ldr, rows, C, F, yp, ldy, zp, ldz, wp, wn,
                         _stream(here)))
    return {"y": y, "z": z}


def gc_linear_backward(dy, x, W, N: int, n_c: int, z=None, act: int = GC_ACT_NONE, dx=True, G=True, Gb=True,
                       ws: Workspace | None = None):
    """Gradient of gc_linear from dy (N n_c x F, of y).  Returns dict with dx (x's type), G (N x F C float32:
    per chunk the gradient of W, un-normalised) and Gb (N x F float32: of the bias); booleans ask for an
    output, tensors are written into (G and Gb may be column slices of a larger matrix).  The gradient of the
    residual is dy."""
    xt, wt = _elt(x, "x"), _elt(W, "W")
    T, C = x.shape
    F = W.shape[0]
    if T != N * n_c:
        raise ValueError("x must have N * n_c rows")
    dt, dev = x.dtype, x.device
    yp, lddy = _rows(dy, dt, "dy", (T, F))
    zp, ldz = _rows(z, dt, "z", (T, F))
    xp, ldx = _rows(x, dt, "x", (T, C))
    wp_, ldw = _rows(W, W.dtype, "W", (F, C))
    dx, dp, lddx = _out(dx, T, C, dt, dev, "dx")
    G, gp, ldg = _out(G, N, F * C, torch.float32, dev, "G")
    Gb, bp, ldgb = _out(Gb, N, F, torch.float32, dev, "Gb")
    here = _same_device(dy, x, W, z, dx, G, Gb)
    e = 4 - 2 * xt
    want = (dx is not None) + 2 * (G is not None) + 4 * (Gb is not None)
    ws, (wp, wn) = _ws(ws, _device_bytes(here, "gc_linear_backward_workspace", N, n_c, C, F, xt, wt, act,
                                        _on_16(xp, ldx, T, e), _on_16(wp_, ldw, F, 4 - 2 * wt), _on_16(yp, lddy, T, e),
                                        want), dev)
    _check(lib.gc_linear_backward(yp, lddy, zp, ldz, xp, ldx, xt, wp_, ldw, wt, act, N, n_c, C, F, dp, lddx, gp, ldg,
                                  bp, ldgb, wp, wn, _stream(here)))
    return {"dx": dx, "G": G, "Gb": Gb}


# ---------------------------------------------------------------- orthogonalised updates
def _mats(t, dtype, name, shape):
    """(device pointer, row stride, matrix stride) of a CUDA matrix, or of a batch of them."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA tensor")
    if t.dtype is not dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if t.shape != shape:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    if t.stride(-1) != 1 and shape[-1] > 1:
        raise ValueError(f"the elements of a row of {name} must lie next to each other")
    ld = t.stride(-2) if shape[-2] > 1 else shape[-1]
    return t.data_ptr(), ld, t.stride(0) if len(shape) == 3 else 0


def _mats_of(t, name):
    """(batch, rows, cols, element type) of a matrix or of a batch of them."""
    if not isinstance(t, torch.Tensor) or t.dim() not in (2, 3):
        raise TypeError(f"{name} must be a matrix or a batch of matrices")
    if t.dtype not in (torch.float32, torch.bfloat16):
        raise TypeError(f"{name} must be float32 or bfloat16")
    return (t.shape[0] if t.dim() == 3 else 1, t.shape[-2], t.shape[-1], GC_BF16 if t.dtype is torch.bfloat16 else GC_F32)


def _coeffs(coeffs):
    """Host array of the polynomial's three coefficients (None -> NULL)."""
    if coeffs is None:
        return None
    if len(coeffs) != 3:
        raise ValueError("coeffs must be three numbers")
    return (ctypes.c_float * 3)(*coeffs)


def gc_orthogonalize(u, coeffs=None, steps: int = 5, eps: float = 1e-7, out=None, ws: Workspace | None = None):
    """u (rows x cols, or batch x rows x cols; float32 or bfloat16) with its singular values drawn towards 1 by
    `steps` Newton-Schulz products, X <- (a + b X X^T + c (X X^T)^2) X from u / max(|u|, eps).  Returns
    out, which may be u."""
    batch, rows, cols, dt = _mats_of(u, "u")
    if out is None:
        out = torch.empty(u.shape, dtype=u.dtype, device=u.device)
    up, ldu, su = _mats(u, u.dtype, "u", u.shape)
    op, ldo, so = _mats(out, u.dtype, "out", u.shape)
    here = _same_device(u, out)
    ws, (wp, wn) = _ws(ws, _device_bytes(here, "gc_orthogonalize_workspace", batch, rows, cols, dt), u.device)
    _check(lib.gc_orthogonalize(up, ldu, su, dt, batch, rows, cols, _coeffs(coeffs), steps, eps, op, ldo, so, wp, wn,
                                _stream(here)))
    return out


def gc_muon_step(w, momentum, g, lr: float, Ntil: int, mu: float = 0.95, nesterov: bool = True,
                 weight_decay: float = 0.0, scale: float = 1.0, coeffs=None, steps: int = 5, eps: float = 1e-7,
                 ws: Workspace | None = None) -> None:
    """momentum = mu momentum + g / Ntil; w = (1 - lr weight_decay) w - lr scale O, in place, with O the
    orthogonalised momentum (of g / Ntil + mu momentum where nesterov).  w, momentum, g: float32, rows x cols or
    batch x rows x cols, their rows strided as they may be."""
    batch, rows, cols, _ = _mats_of(w, "w")
    wp_, ldw, sw = _mats(w, torch.float32, "w", w.shape)
    mp, ldm, sm = _mats(momentum, torch.float32, "momentum", w.shape)
    gp, ldg, sg = _mats(g, torch.float32, "g", w.shape)
    here = _same_device(w, momentum, g)
    ws, (wp, wn) = _ws(ws, _device_bytes(here, "gc_orthogonalize_workspace", batch, rows, cols, GC_F32), w.device)
    _check(lib.gc_muon_step(wp_, ldw, sw, mp, ldm, sm, gp, ldg, sg, batch, rows, cols, lr, Ntil, mu, int(nesterov),
                            weight_decay, scale, _coeffs(coeffs), steps, eps, wp, wn, _stream(here)))


# ---------------------------------------------------------------- Algorithm 1
def gc_coeff_workspace(N, m, delta, ell, npat):
    return lib.gc_coeff_workspace(N, m, delta, ell, npat)


def gc_find_encoding_coeff(R, ell, order, N, m, delta, psi, E=True, C=True, delta_out=True,
                           support=False, coef_err=True, est=True, ws: Workspace | None = None):
    """Batched Algorithm 1.  Boolean arguments request an output (allocated
    here); tensors are used as given.  Returns a dict of the outputs."""
    npat = psi.shape[0]
    dev = psi.device

    def out(flag, shape, dtype):
        if isinstance(flag, torch.Tensor):
            return flag
        return torch.empty(shape, dtype=dtype, device=dev) if flag else None

    res = {
        "E": out(E, (npat, m, delta, ell), torch.float64),
        "C": out(C, (npat, ell, N * ell), torch.float32),
        "delta": out(delta_out, (npat, N), torch.uint8),
        "support": out(support, (npat, N, m), torch.uint8),
        "coef_err": out(coef_err, (npat,), torch.float64),
        "est": out(est, (npat,), torch.float64),
    }
    ws, (wp, wn) = _ws(ws, _bytes("gc_coeff_workspace", N, m, delta, ell, npat), dev)
    _check(lib.gc_find_encoding_coeff(
        _dev(R, torch.float64, "R", (ell, m)), ell, _dev(order, torch.int32, "order", (m, delta)),
        N, m, delta, _dev(psi, torch.int32, "psi", (npat, m)), npat,
        _dev(res["E"], torch.float64, "E"), _dev(res["C"], torch.float32, "C"),
        _dev(res["delta"], torch.uint8, "delta_out"), _dev(res["support"], torch.uint8, "support"),
        _dev(res["coef_err"], torch.float64, "coef_err"), _dev(res["est"], torch.float64, "est"),
        wp, wn, _stream()))
    return res


# ---------------------------------------------------------------- encode / decode
def gc_encode_workspace(N, m, delta, ell, npat, d):
    return lib.gc_encode_workspace(N, m, delta, ell, npat, d)


def gc_encode(R, ell, order, N, m, delta, psi, G, T=None, ws: Workspace | None = None):
    """Worker transmissions T (npat x m x L float32), eq. (2)."""
    npat = psi.shape[0]
    d = G.shape[1]
    L = block_length(d, ell)
    if T is None:
        T = torch.empty(npat, m, L, dtype=torch.float32, device=G.device)
    ws, (wp, wn) = _ws(ws, _bytes("gc_encode_workspace", N, m, delta, ell, npat, d), G.device)
    _check(lib.gc_encode(_dev(R, torch.float64, "R", (ell, m)), ell,
                         _dev(order, torch.int32, "order", (m, delta)), N, m, delta,
                         _dev(psi, torch.int32, "psi", (npat, m)), npat,
                         _dev(G, torch.float32, "G", (N, d)), d,
                         _dev(T, torch.float32, "T", (npat, m, L)), wp, wn, _stream()))
    return T


def gc_encode_with_coeffs(E, ell, order, N, m, delta, psi, G, T=None):
    """Eq. (2) alone: transmissions from Algorithm 1's coefficients E
    (npat x m x delta x ell float64, as gc_find_encoding_coeff returns)."""
    npat = psi.shape[0]
    d = G.shape[1]
    L = block_length(d, ell)
    if T is None:
        T = torch.empty(npat, m, L, dtype=torch.float32, device=G.device)
    _check(lib.gc_encode_with_coeffs(_dev(E, torch.float64, "E", (npat, m, delta, ell)), ell,
                                     _dev(order, torch.int32, "order", (m, delta)), N, m, delta,
                                     _dev(psi, torch.int32, "psi", (npat, m)), npat,
                                     _dev(G, torch.float32, "G", (N, d)), d,
                                     _dev(T, torch.float32, "T", (npat, m, L)), _stream()))
    return T


def gc_decode_tx(R, ell, m, T, d, ghat=None):
    """PS decode of transmissions: ghat (npat x d float32)."""
    npat = T.shape[0]
    L = block_length(d, ell)
    if ghat is None:
        ghat = torch.empty(npat, d, dtype=torch.float32, device=T.device)
    _check(lib.gc_decode_tx(_dev(R, torch.float64, "R", (ell, m)), ell, m,
                            _dev(T, torch.float32, "T", (npat, m, L)), npat, d,
                            _dev(ghat, torch.float32, "ghat", (npat, d)), _stream()))
    return ghat


def gc_decode_batch_workspace(N, m, delta, ell, npat, d):
    return lib.gc_decode_batch_workspace(N, m, delta, ell, npat, d)


def gc_decode_batch(R, ell, order, N, m, delta, psi, G, Ghat=True, coef_err=True, est=True,
                    grad_mse=True, ws: Workspace | None = None):
    """Batched decode-combine.  Returns dict with Ghat (npat x d float32 or
    None), coef_err, est, grad_mse (npat float64 or None)."""
    npat = psi.shape[0]
    d = G.shape[1]
    dev = G.device

    def out(flag, shape, dtype):
        if isinstance(flag, torch.Tensor):
            return flag
        return torch.empty(shape, dtype=dtype, device=dev) if flag else None

    res = {
        "Ghat": out(Ghat, (npat, d), torch.float32),
        "coef_err": out(coef_err, (npat,), torch.float64),
        "est": out(est, (npat,), torch.float64),
        "grad_mse": out(grad_mse, (npat,), torch.float64),
    }
    ws, (wp, wn) = _ws(ws, _bytes("gc_decode_batch_workspace", N, m, delta, ell, npat, d), dev)
    _check(lib.gc_decode_batch(
        _dev(R, torch.float64, "R", (ell, m)), ell, _dev(order, torch.int32, "order", (m, delta)),
        N, m, delta, _dev(psi, torch.int32, "psi", (npat, m)), npat,
        _dev(G, torch.float32, "G", (N, d)), d, _dev(res["Ghat"], torch.float32, "Ghat", (npat, d)),
        _dev(res["coef_err"], torch.float64, "coef_err"), _dev(res["est"], torch.float64, "est"),
        _dev(res["grad_mse"], torch.float64, "grad_mse"), wp, wn, _stream()))
    return res


def gc_decode_plan(R, ell, order, N, m, delta, psi, plan=None, coef_err=True, est=True,
                   ws: Workspace | None = None):
    """Algorithm 1 for every pattern into an opaque plan (uint8 device tensor)
    for gc_decode_apply.  Returns dict with plan, coef_err, est."""
    npat = psi.shape[0]
    dev = psi.device
    nb = _bytes("gc_decode_plan_bytes", N, ell, npat)
    if plan is None:
        plan = torch.empty(max(int(nb), 256), dtype=torch.uint8, device=dev)
    ce = coef_err if isinstance(coef_err, torch.Tensor) else (
        torch.empty(npat, dtype=torch.float64, device=dev) if coef_err else None)
    es = est if isinstance(est, torch.Tensor) else (
        torch.empty(npat, dtype=torch.float64, device=dev) if est else None)
    ws, (wp, wn) = _ws(ws, _bytes("gc_decode_plan_workspace", N, m, delta, ell, npat), dev)
    _check(lib.gc_decode_plan(_dev(R, torch.float64, "R", (ell, m)), ell,
                              _dev(order, torch.int32, "order", (m, delta)), N, m, delta,
                              _dev(psi, torch.int32, "psi", (npat, m)), npat,
                              _dev(plan, torch.uint8, "plan"), plan.numel(),
                              _dev(ce, torch.float64, "coef_err"), _dev(es, torch.float64, "est"),
                              wp, wn, _stream()))
    return {"plan": plan, "coef_err": ce, "est": es}


def gc_decode_prepare(R, ell, order, N, m, delta, prep=None):
    """Holders and the Algorithm 1 memo table for (R, assignment), once:
    a uint8 device buffer for gc_decode_plan_prepared."""
    nb = int(lib.gc_decode_prepare_bytes(N, m, delta, ell))
    if nb == 0:
        raise ValueError("unsupported shape for gc_decode_prepare")
    if prep is None:
        prep = torch.empty(nb, dtype=torch.uint8, device=R.device)
    _check(lib.gc_decode_prepare(_dev(R, torch.float64, "R", (ell, m)), ell,
                                 _dev(order, torch.int32, "order", (m, delta)), N, m, delta,
                                 _dev(prep, torch.uint8, "prep"), prep.numel(), _stream()))
    return prep


def gc_decode_plan_prepared(prep, R, ell, N, m, delta, psi, plan=None, coef_err=True, est=True,
                            ws: Workspace | None = None):
    """gc_decode_plan from a gc_decode_prepare buffer.  Returns dict with
    plan, coef_err, est."""
    npat = psi.shape[0]
    dev = psi.device
    nb = _bytes("gc_decode_plan_bytes", N, ell, npat)
    if plan is None:
        plan = torch.empty(max(int(nb), 256), dtype=torch.uint8, device=dev)
    ce = coef_err if isinstance(coef_err, torch.Tensor) else (
        torch.empty(npat, dtype=torch.float64, device=dev) if coef_err else None)
    es = est if isinstance(est, torch.Tensor) else (
        torch.empty(npat, dtype=torch.float64, device=dev) if est else None)
    ws, (wp, wn) = _ws(ws, _bytes("gc_decode_plan_prepared_workspace"), dev)
    _check(lib.gc_decode_plan_prepared(_dev(prep, torch.uint8, "prep"),
                                       _dev(R, torch.float64, "R", (ell, m)), ell, N, m, delta,
                                       _dev(psi, torch.int32, "psi", (npat, m)), npat,
                                       _dev(plan, torch.uint8, "plan"), plan.numel(),
                                       _dev(ce, torch.float64, "coef_err"),
                                       _dev(es, torch.float64, "est"), wp, wn, _stream()))
    return {"plan": plan, "coef_err": ce, "est": es}


def gc_decode_apply(plan, ell, N, npat, G, Ghat=True, grad_mse=True, ws: Workspace | None = None):
    """Ghat (npat x d) and/or grad_mse (npat) from a gc_decode_plan plan and G."""
    d = G.shape[1]
    dev = G.device
    if not isinstance(Ghat, torch.Tensor):
        Ghat = torch.empty(npat, d, dtype=torch.float32, device=dev) if Ghat else None
    if not isinstance(grad_mse, torch.Tensor):
        grad_mse = torch.empty(npat, dtype=torch.float64, device=dev) if grad_mse else None
    ws, (wp, wn) = _ws(ws, _bytes("gc_decode_apply_workspace", N, ell, npat, d), dev)
    _check(lib.gc_decode_apply(_dev(plan, torch.uint8, "plan"), ell, N, npat,
                               _dev(G, torch.float32, "G", (N, d)), d,
                               _dev(Ghat, torch.float32, "Ghat", (npat, d)),
                               _dev(grad_mse, torch.float64, "grad_mse"), wp, wn, _stream()))
    return {"Ghat": Ghat, "grad_mse": grad_mse}


def gc_set_wait_limit(cycles: int) -> None:
    """Testing aid: device waits give up after `cycles` clock cycles (0 = default)."""
    _check(lib.gc_set_wait_limit(int(cycles)))


GC_STALL_CHUNK_GRADS = 1
GC_STALL_COMBINE = 2
GC_STALL_BATCHED = 4
GC_STALL_XENT = 16
GC_STALL_LINEAR = 32
GC_STALL_MUON = 64


def gc_inject_stall(kernels: int) -> None:
    """Testing aid: the next launch of each selected kernel withholds its copies."""
    _check(lib.gc_inject_stall(int(kernels)))


GC_DECODE_AUTO = 0
GC_DECODE_DENSE = 1
GC_DECODE_RESIDUAL = 2


def gc_set_decode_policy(policy: int) -> None:
    """Path of the batched decode per pattern: GC_DECODE_AUTO (default),
    GC_DECODE_DENSE (tensor-core GEMM) or GC_DECODE_RESIDUAL (sum of the
    chunk gradients plus the non-identity blocks).  Process-wide."""
    _check(lib.gc_set_decode_policy(int(policy)))


def gc_kernel_launches() -> int:
    return int(lib.gc_kernel_launches())


def gc_decode_combine_workspace(N, ell, npat, d):
    return lib.gc_decode_combine_workspace(N, ell, npat, d)


def gc_decode_combine(C, ell, N, G, Ghat=True, grad_mse=True, ws: Workspace | None = None):
    """Ghat (npat x d) = C . G for a decode matrix C (npat x ell x N*ell) from
    gc_find_encoding_coeff; grad_mse optional."""
    npat = C.shape[0]
    d = G.shape[1]
    dev = G.device
    if not isinstance(Ghat, torch.Tensor):
        Ghat = torch.empty(npat, d, dtype=torch.float32, device=dev) if Ghat else None
    if not isinstance(grad_mse, torch.Tensor):
        grad_mse = torch.empty(npat, dtype=torch.float64, device=dev) if grad_mse else None
    ws, (wp, wn) = _ws(ws, _bytes("gc_decode_combine_workspace", N, ell, npat, d), dev)
    _check(lib.gc_decode_combine(_dev(C, torch.float32, "C", (npat, ell, N * ell)), ell, N, npat,
                                 _dev(G, torch.float32, "G", (N, d)), d,
                                 _dev(Ghat, torch.float32, "Ghat", (npat, d)),
                                 _dev(grad_mse, torch.float64, "grad_mse"), wp, wn, _stream()))
    return {"Ghat": Ghat, "grad_mse": grad_mse}


def gc_mse_workspace(N, m, delta, ell, npat, d):
    return lib.gc_mse_workspace(N, m, delta, ell, npat, d)


def gc_mse(R, ell, order, N, m, delta, psi, G, coef_err=True, est=True, grad_mse=True,
           ws: Workspace | None = None):
    """Error measures only; decoded gradients are never written."""
    npat = psi.shape[0]
    d = G.shape[1]
    dev = G.device

    def out(flag, shape, dtype):
        if isinstance(flag, torch.Tensor):
            return flag
        return torch.empty(shape, dtype=dtype, device=dev) if flag else None

    res = {
        "coef_err": out(coef_err, (npat,), torch.float64),
        "est": out(est, (npat,), torch.float64),
        "grad_mse": out(grad_mse, (npat,), torch.float64),
    }
    ws, (wp, wn) = _ws(ws, _bytes("gc_mse_workspace", N, m, delta, ell, npat, d), dev)
    _check(lib.gc_mse(
        _dev(R, torch.float64, "R", (ell, m)), ell, _dev(order, torch.int32, "order", (m, delta)),
        N, m, delta, _dev(psi, torch.int32, "psi", (npat, m)), npat,
        _dev(G, torch.float32, "G", (N, d)), d, _dev(res["coef_err"], torch.float64, "coef_err"),
        _dev(res["est"], torch.float64, "est"), _dev(res["grad_mse"], torch.float64, "grad_mse"),
        wp, wn, _stream()))
    return res


def gc_sgd_step(w, ghat, lr: float, Ntil: int):
    """w -= lr * ghat / N~ in place."""
    d = w.shape[0]
    _check(lib.gc_sgd_step(_dev(w, torch.float32, "w", (d,)), _dev(ghat, torch.float32, "ghat", (d,)),
                           d, float(lr), int(Ntil), _stream()))
    return w


def gc_live_step(E, R, ell, order, N, m, delta, psi, G, w, lr: float, Ntil: int, T=None, ghat=None):
    """One live realization in one launch: eq. (2) transmissions, their PS
    decode and the update of w (in place).  E is the pattern's m x delta x ell
    float64 coefficients (a 1 x m x delta x ell batch is accepted), psi its m
    processed counts; T (m x L) and ghat (d) are written when given."""
    d = G.shape[1]
    L = block_length(d, ell)

    def as_shape(t, shape):
        return t if t is None or t.shape == shape else t.reshape(shape)
    E, psi = as_shape(E, (m, delta, ell)), as_shape(psi, (m,))
    T, ghat = as_shape(T, (m, L)), as_shape(ghat, (d,))
    _check(lib.gc_live_step(_dev(E, torch.float64, "E", (m, delta, ell)),
                            _dev(R, torch.float64, "R", (ell, m)), ell,
                            _dev(order, torch.int32, "order", (m, delta)), N, m, delta,
                            _dev(psi, torch.int32, "psi", (m,)),
                            _dev(G, torch.float32, "G", (N, d)), d, float(lr), int(Ntil),
                            _dev(w, torch.float32, "w", (d,)),
                            _dev(T, torch.float32, "T", (m, L)),
                            _dev(ghat, torch.float32, "ghat", (d,)), _stream()))
    return w
