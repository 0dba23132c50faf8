"""Measured cases of the language-model operators: what a coded training step does at the output
end of a language model, and what scoring does there with one token or a few thousand.

Five kinds, two or more cases each:

  dropout    out = residual + D(x): a mask drawn from (seed, offset, row, column), never stored
  norm       h = residual + D(x), y = layer norm of h, with the statistics of every row
  norm_grad  the gradient of that: of the branch, of the residual, and per chunk of rows of gamma, beta
  head       losses and log-sum-exp of softmax cross entropy over the vocabulary, for scoring
  head_grad  the same with its gradient: of the rows, and per chunk of the vocabulary's matrix

Rows are points (tokens); chunk i of N is rows [i n_c, (i+1) n_c), and gradients of parameters are
kept per chunk, un-normalised, since they are what a gradient code encodes.
"""
import math

import numpy as np
import torch

own = False

_DEV = "cuda"
_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
_BYTES = {"f32": 4, "bf16": 2}
_EPS = 1e-5


# ------------------------------------------------------------------------------------ the cases
def listed():
    return [
        # the 6-worker example's 6 x 32 points: launches and latency alone
        dict(name="dropout_tiny", kind="dropout", rows=192, cols=64, x="f32", p=0.1, residual=False),
        # a residual branch of a training batch of 32,768 tokens (805 MB moved)
        dict(name="dropout_batch", kind="dropout", rows=32768, cols=4096, x="bf16", p=0.1, residual=True),
        # one token on its way to the head while serving
        dict(name="norm_token", kind="norm", rows=1, cols=4096, x="bf16", p=0.0, residual=True),
        # a width that is no multiple of any vector, 20 chunks of 333 points
        dict(name="norm_odd", kind="norm", rows=6660, cols=1001, x="f32", p=0.0, residual=False),
        # the last block of a training batch: branch with dropout, residual, norm (537 MB moved)
        dict(name="norm_batch", kind="norm", rows=16384, cols=4096, x="bf16", p=0.1, residual=True),
        # gradient of the 6-worker example
        dict(name="norm_grad_tiny", kind="norm_grad", N=6, n_c=32, cols=64, x="f32", p=0.0, residual=False),
        # gradient of norm_batch, eight chunks
        dict(name="norm_grad_batch", kind="norm_grad", N=8, n_c=2048, cols=4096, x="bf16", p=0.1, residual=True),
        # the loss of one token: one pass over a vocabulary of 65,536 rows (268 MB)
        dict(name="head_token", kind="head", N=1, n_c=1, C=2048, V=65536, x="bf16", w="bf16"),
        # perplexity of a document of 2,048 tokens
        dict(name="head_score", kind="head", N=1, n_c=2048, C=1024, V=32000, x="bf16", w="bf16"),
        # one coded step of the 6-worker example with a toy vocabulary, in 32 bits
        dict(name="head_grad_tiny", kind="head_grad", N=6, n_c=32, C=64, V=257, x="f32", w="f32"),
        # odd sizes throughout; the weights are a slice of the 32-bit parameter vector
        dict(name="head_grad_ragged", kind="head_grad", N=20, n_c=77, C=1000, V=10007, x="bf16", w="f32"),
        # a coded training step over 8,192 tokens in eight chunks (4.3 GB of chunk gradients)
        dict(name="head_grad_batch", kind="head_grad", N=8, n_c=1024, C=2048, V=65536, x="bf16", w="bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A width: as it falls, or rounded to a multiple of 8 or 64, as most models' are."""
    w = _log(rng, lo, hi)
    m = rng.choice([1, 8, 64])
    return max(lo, w // m * m)


def draw(rng):
    kind = rng.choice(["dropout", "norm", "norm_grad", "head", "head_grad", "head_grad"])
    x = rng.choice(["f32", "bf16", "bf16"])
    p = rng.choice([0.0, 0.05, 0.1, 0.3])
    if kind == "dropout":
        cols = _width(rng, 64, 8192)
        rows = _log(rng, 1, min(32768, (1 << 27) // cols))
        return dict(kind=kind, rows=rows, cols=cols, x=x, p=rng.choice([0.05, 0.1, 0.5]),
                    residual=rng.random() < 0.5)
    if kind == "norm":
        cols = _width(rng, 64, 8192)
        rows = _log(rng, 1, min(32768, (1 << 26) // cols))
        return dict(kind=kind, rows=rows, cols=cols, x=x, p=p, residual=p > 0 or rng.random() < 0.5)
    if kind == "norm_grad":
        cols = _width(rng, 64, 8192)
        N = _log(rng, 1, 64)
        n_c = _log(rng, 1, max(2, min(4096, (1 << 26) // (cols * N))))
        return dict(kind=kind, N=N, n_c=n_c, cols=cols, x=x, p=p, residual=p > 0 or rng.random() < 0.5)
    w = rng.choice(["f32", "bf16"]) if x == "bf16" else "f32"
    C = _width(rng, 64, 2048)
    V = _width(rng, 257, 65536)
    if kind == "head":
        n_c = _log(rng, 1, 8192)
        return dict(kind=kind, N=1, n_c=n_c, C=C, V=V, x=x, w=w)
    N = _log(rng, 1, 32)
    while N > 1 and N * V * C > 1 << 30:
        N //= 2
    n_c = _log(rng, 1, max(2, 8192 // N))
    return dict(kind=kind, N=N, n_c=n_c, C=C, V=V, x=x, w=w)


# ------------------------------------------------------------------------------------ the inputs
def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device=_DEV, dtype=torch.float32)


def prepare(case, seed):
    c = dict(case)
    kind = c["kind"]
    g = torch.Generator(device=_DEV).manual_seed(int(seed) + 1)
    xt = _TYPES[c["x"]]
    # the generator's key and the number of the draw, as a training loop counts them
    s = dict(case=c, key=(int(seed) * 0x9E3779B97F4A7C15 + 12345) % (1 << 63), offset=int(seed) % 100003)
    if kind in ("dropout", "norm", "norm_grad"):
        rows = c["rows"] if "rows" in c else c["N"] * c["n_c"]
        cols = c["cols"]
        if kind != "norm_grad":
            s["x"] = _randn(g, rows, cols).to(xt)
            s["residual"] = (1.5 * _randn(g, rows, cols) + 0.25).to(xt) if c["residual"] else None
        if kind != "dropout":
            s["gamma"] = 1 + 0.2 * _randn(g, cols)
        if kind == "norm":
            s["beta"] = 0.2 * _randn(g, cols)
        if kind == "norm_grad":
            h = (1.5 * _randn(g, rows, cols) + 0.25).to(xt)
            f = h.float()
            s["h"], s["mean"] = h, f.mean(1)
            s["rstd"] = torch.rsqrt((f - s["mean"][:, None]).square().mean(1) + _EPS)
            s["dy"] = _randn(g, rows, cols).to(xt)
            s["dh"] = _randn(g, rows, cols).to(xt) if c["residual"] else None
        return s
    T, C, V = c["N"] * c["n_c"], c["C"], c["V"]
    s["X"] = _randn(g, T, C).to(xt)                              # rows out of a layer norm
    s["W"] = (_randn(g, V, C) * (2 / math.sqrt(C))).to(_TYPES[c["w"]])   # logits of spread 2
    # tokens: frequent ones more often than rare ones; of several, some are padding (a negative label)
    u = torch.rand(T, generator=g, device=_DEV, dtype=torch.float64)
    y = (torch.exp(u * math.log(V + 1.0)) - 1).long().clamp_(0, V - 1)
    if T > 1:
        y = torch.where(torch.rand(T, generator=g, device=_DEV) < 0.0625, torch.full_like(y, -100), y)
    s["y"] = y
    return s


# ------------------------------------------------------------------------------------ the calls
_scratch = []


def _workspace(gc):
    """The program's one workspace, as the library's users keep it."""
    if not _scratch:
        _scratch.append(gc.Workspace())
    return _scratch[0]


def run(state):
    c = state["case"]
    kind = c["kind"]
    if not own:
        return _PLAIN[kind](state, c)
    import paper_2405_19509_gb300 as gc
    if kind == "dropout":
        return {"out": gc.gc_dropout(state["x"], c["p"], state["key"], state["offset"],
                                     residual=state["residual"])}
    if kind == "norm":
        r = gc.gc_layer_norm(state["x"], state["gamma"], state["beta"], _EPS,
                             residual=state["residual"], p=c["p"], seed=state["key"],
                             offset=state["offset"])
        return {k: r[k] for k in (("y", "mean", "rstd", "h") if c["residual"] else ("y", "mean", "rstd"))}
    ws = _workspace(gc)
    if kind == "norm_grad":
        r = gc.gc_layer_norm_backward(state["dy"], state["h"], state["mean"], state["rstd"],
                                      state["gamma"], c["N"], c["n_c"], dh=state["dh"], p=c["p"],
                                      seed=state["key"], offset=state["offset"],
                                      dresidual=c["residual"], ws=ws)
        return {k: r[k] for k in (("dx", "G", "dresidual") if c["residual"] else ("dx", "G"))}
    if kind == "head":
        r = gc.gc_softmax_xent(state["X"], state["W"], state["y"], c["N"], c["n_c"], loss=False,
                               dX=False, G=False, ws=ws)
        return {"row_loss": r["row_loss"], "lse": r["lse"]}
    r = gc.gc_softmax_xent(state["X"], state["W"], state["y"], c["N"], c["n_c"], loss=False, ws=ws)
    return {k: r[k] for k in ("row_loss", "lse", "dX", "G")}


# ------------------------------------------------------------------------------------ plain forms
def _keep(rows, cols, p, key, offset):
    """(keep mask, scale): 16-bit numbers from Philox4x32-10, eight to a counter.  The counter is
    (row ceil(cols / 8) + column / 8, offset), the key the seed."""
    t = min(int(p * 65536 + 0.5), 65535)
    groups = (cols + 7) // 8
    m = 0xFFFFFFFF
    e = torch.arange(rows * groups, device=_DEV, dtype=torch.int64)
    x0, x1 = e & m, e >> 32
    x2, x3 = torch.full_like(e, offset & m), torch.full_like(e, (offset >> 32) & m)
    k0, k1 = key & m, (key >> 32) & m
    for _ in range(10):
        a, b = x0 * 0xD2511F53, x2 * 0xCD9E8D57  # the low 64 bits: nothing is lost below 2^64
        x0, x1, x2, x3 = ((b >> 32) & m) ^ x1 ^ k0, b & m, ((a >> 32) & m) ^ x3 ^ k1, a & m
        k0, k1 = (k0 + 0x9E3779B9) & m, (k1 + 0xBB67AE85) & m
    u = torch.stack([x0 & 0xFFFF, x0 >> 16, x1 & 0xFFFF, x1 >> 16, x2 & 0xFFFF, x2 >> 16, x3 & 0xFFFF, x3 >> 16], 1)
    return (u >= t).view(rows, groups * 8)[:, :cols], 65536.0 / (65536 - t)


def _drop(x, c, state):
    if c["p"] == 0:
        return x
    keep, scale = _keep(x.shape[0], x.shape[1], c["p"], state["key"], state["offset"])
    return torch.where(keep, x * scale, torch.zeros((), device=_DEV))


def _plain_dropout(state, c):
    out = _drop(state["x"].float(), c, state)
    if state["residual"] is not None:
        out = out + state["residual"].float()
    return {"out": out.to(state["x"].dtype)}


def _plain_norm(state, c):
    h = _drop(state["x"].float(), c, state)
    if state["residual"] is not None:
        h = h + state["residual"].float()
    mean = h.mean(1)
    d = h - mean[:, None]
    rstd = torch.rsqrt(d.square().mean(1) + _EPS)
    y = d * rstd[:, None] * state["gamma"] + state["beta"]
    t = state["x"].dtype
    r = {"y": y.to(t), "mean": mean, "rstd": rstd}
    return dict(r, h=h.to(t)) if c["residual"] else r


def _plain_norm_grad(state, c):
    dy, t = state["dy"].float(), state["dy"].dtype
    n = (state["h"].float() - state["mean"][:, None]) * state["rstd"][:, None]
    a = dy * state["gamma"]
    d = state["rstd"][:, None] * (a - a.mean(1, keepdim=True) - n * (a * n).mean(1, keepdim=True))
    if state["dh"] is not None:
        d = d + state["dh"].float()
    shape = (c["N"], c["n_c"], c["cols"])
    G = torch.cat([(dy * n).view(shape).sum(1), dy.view(shape).sum(1)], 1)
    r = {"dx": _drop(d, c, state).to(t), "G": G}
    return dict(r, dresidual=d.to(t)) if c["residual"] else r


def _plain_head(state, c):
    z = state["X"].float() @ state["W"].float().T
    top = z.amax(1)
    lse = top + torch.log(torch.exp(z - top[:, None]).sum(1))
    y = state["y"]
    at = z.gather(1, y.clamp_min(0)[:, None])[:, 0]
    r = {"row_loss": torch.where(y >= 0, lse - at, torch.zeros_like(lse)), "lse": lse}
    return r, z


def _plain_head_grad(state, c):
    r, z = _plain_head(state, c)
    y = state["y"]
    live = (y >= 0).float()[:, None]
    P = torch.exp(z - r["lse"][:, None]) * live
    P.scatter_add_(1, y.clamp_min(0)[:, None], -live)
    X, W = state["X"].float(), state["W"].float()
    G = torch.bmm(P.view(c["N"], c["n_c"], c["V"]).transpose(1, 2), X.view(c["N"], c["n_c"], c["C"]))
    return dict(r, dX=(P @ W).to(state["X"].dtype), G=G.view(c["N"], -1))


_PLAIN = {"dropout": _plain_dropout, "norm": _plain_norm, "norm_grad": _plain_norm_grad,
          "head": lambda s, c: _plain_head(s, c)[0], "head_grad": _plain_head_grad}


# ------------------------------------------------------------------------------------ the work
def work(case):
    """Bytes: inputs read once, outputs written once.  Operations: the products; of the head's gradient
    three of them (logits, rows, matrix), though keeping no logits takes the first one twice."""
    c, e = case, _BYTES[case["x"]]
    kind = c["kind"]
    if kind == "dropout":
        n = c["rows"] * c["cols"]
        return {"bytes": n * e * (3 if c["residual"] else 2), "flops": n * 2}
    if kind == "norm":
        n = c["rows"] * c["cols"]
        return {"bytes": n * e * (4 if c["residual"] else 2) + 8 * c["cols"] + 8 * c["rows"], "flops": 8 * n}
    if kind == "norm_grad":
        n = c["N"] * c["n_c"] * c["cols"]
        return {"bytes": n * e * (5 if c["residual"] else 3) + 8 * c["N"] * c["n_c"] + 4 * c["cols"] + 8 * c["N"] * c["cols"],
                "flops": 14 * n}
    T, C, V = c["N"] * c["n_c"], c["C"], c["V"]
    read = T * C * e + V * C * _BYTES[c["w"]] + 8 * T
    if kind == "head":
        return {"bytes": read + 8 * T, "flops": 2 * T * V * C}
    return {"bytes": read + 8 * T + T * C * e + 4 * c["N"] * V * C, "flops": 6 * T * V * C}


# ------------------------------------------------------------------------------------ 64 bits
def _mask64(rows, cols, p, key, offset):
    """The factor of every element (0 or 1 / (1 - p)), with NumPy's unsigned 64-bit numbers."""
    t = np.uint64(min(int(p * 65536 + 0.5), 65535))
    groups = -(-cols // 8)
    low, half = np.uint64(0xFFFFFFFF), np.uint64(32)
    at = np.arange(rows * groups, dtype=np.uint64)
    w = [at & low, at >> half, np.uint64(offset & 0xFFFFFFFF), np.uint64(offset >> 32)]
    k = [key & 0xFFFFFFFF, (key >> 32) & 0xFFFFFFFF]
    for _ in range(10):
        left, right = w[0] * np.uint64(0xD2511F53), w[2] * np.uint64(0xCD9E8D57)
        w = [(right >> half) ^ w[1] ^ np.uint64(k[0]), right & low, (left >> half) ^ w[3] ^ np.uint64(k[1]), left & low]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    f = np.empty((rows * groups, 8), np.bool_)
    for j in range(8):
        f[:, j] = ((w[j // 2] >> np.uint64(16 * (j % 2))) & np.uint64(0xFFFF)) >= t
    f = torch.from_numpy(f.reshape(rows, groups * 8)).to(_DEV)[:, :cols]
    return f.double() * (65536.0 / (65536.0 - float(t)))


def exact(case, seed):
    s, c = prepare(case, seed), dict(case)
    kind = c["kind"]
    f = None
    if c.get("p"):
        rows = c["rows"] if "rows" in c else c["N"] * c["n_c"]
        f = _mask64(rows, c["cols"], c["p"], s["key"], s["offset"])
    if kind in ("dropout", "norm"):
        h = s["x"].double()
        if f is not None:
            h *= f
        if c["residual"]:
            h += s["residual"].double()
        if kind == "dropout":
            return {"out": h}
        var, mean = torch.var_mean(h, dim=1, correction=0, keepdim=True)
        y = (h - mean) / (var + _EPS).sqrt() * s["gamma"].double() + s["beta"].double()
        r = {"y": y, "mean": mean[:, 0], "rstd": (var[:, 0] + _EPS) ** -0.5}
        return dict(r, h=h) if c["residual"] else r
    if kind == "norm_grad":
        dy, rstd = s["dy"].double(), s["rstd"].double()[:, None]
        n = (s["h"].double() - s["mean"].double()[:, None]) * rstd
        G = torch.stack([(dy * n).unflatten(0, (c["N"], c["n_c"])).sum(1),
                         dy.unflatten(0, (c["N"], c["n_c"])).sum(1)], 1).flatten(1)
        dy *= s["gamma"].double()
        n *= torch.linalg.vecdot(dy, n)[:, None] / c["cols"]
        dy -= dy.sum(1, keepdim=True) / c["cols"] + n
        dy *= rstd
        if c["residual"]:
            dy += s["dh"].double()
        r = {"dx": dy if f is None else dy * f, "G": G}
        return dict(r, dresidual=dy) if c["residual"] else r
    N, n_c, V, C = c["N"], c["n_c"], c["V"], c["C"]
    W, y = s["W"].double(), s["y"]
    dX = torch.empty(N * n_c, C, device=_DEV, dtype=torch.float64)
    G = torch.empty(N, V, C, device=_DEV, dtype=torch.float64) if kind == "head_grad" else None
    losses, lses = [], []
    for i in range(N):
        x, label = s["X"][i * n_c:(i + 1) * n_c].double(), y[i * n_c:(i + 1) * n_c]
        z = torch.einsum("tc,vc->tv", x, W)
        lse = torch.logsumexp(z, 1)
        rows = torch.nonzero(label >= 0)[:, 0]
        loss = torch.zeros_like(lse)
        loss[rows] = lse[rows] - z[rows, label[rows]]
        losses.append(loss)
        lses.append(lse)
        if G is not None:
            z = torch.softmax(z, 1)
            z[rows, label[rows]] -= 1
            z[label < 0] = 0
            dX[i * n_c:(i + 1) * n_c] = z @ W
            G[i] = torch.einsum("tv,tc->vc", z, x)
    r = {"row_loss": torch.cat(losses), "lse": torch.cat(lses)}
    return r if G is None else dict(r, dX=dX, G=G.flatten(1))
