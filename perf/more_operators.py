"""Measured cases of a language model's matrices: the linear layers of its feed-forward blocks, forward and
gradient, and the orthogonalised update of a matrix by its decoded gradient.

Four kinds, two or more cases each:

  linear       y = residual + act(x W^T + b), with z = x W^T + b kept where training wants it
  linear_grad  the gradient of that: of the rows, and per chunk of rows of the matrix and the bias
  ortho        a matrix with its singular values drawn towards 1 by Newton-Schulz products
  muon         momentum of a decoded gradient, orthogonalised, and the update of the matrix

Rows of x are points (tokens); chunk i of N is rows [i n_c, (i+1) n_c), and gradients of parameters are
kept per chunk, un-normalised, since they are what a gradient code encodes.
"""
import math

import torch

own = False

_DEV = "cuda"
_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
_BYTES = {"f32": 4, "bf16": 2}
_COEFF = (3.4445, -4.7750, 2.0315)   # of the quintic whose slope at 0 is the largest that keeps values near 1
_EPS = 1e-7
_MU, _LR, _DECAY = 0.95, 0.02, 0.1


# ------------------------------------------------------------------------------------ the cases
def listed():
    return [
        # the 6-worker example's 6 x 32 points through a toy block: launches and latency alone
        dict(name="linear_tiny", kind="linear", T=192, C=64, F=256, x="f32", w="f32", act="relu",
             bias=True, residual=False, keep=True),
        # one token through the first matrix of a block while serving (34 MB of weights)
        dict(name="linear_token", kind="linear", T=1, C=2048, F=8192, x="bf16", w="bf16", act="gelu",
             bias=True, residual=False, keep=False),
        # a short prompt on odd widths; the weights are a slice of the 32-bit parameter vector
        dict(name="linear_ragged", kind="linear", T=77, C=1000, F=4003, x="bf16", w="f32", act="silu",
             bias=True, residual=False, keep=False),
        # the second matrix of a block over a document of 2,048 tokens, with the residual stream
        dict(name="linear_down", kind="linear", T=2048, C=4096, F=1024, x="bf16", w="bf16", act="none",
             bias=True, residual=True, keep=False),
        # the first matrix over a training batch of 8,192 tokens, z kept for the gradient
        dict(name="linear_batch", kind="linear", T=8192, C=2048, F=8192, x="bf16", w="bf16", act="gelu",
             bias=True, residual=False, keep=True),
        # gradient of linear_tiny
        dict(name="linear_grad_tiny", kind="linear_grad", N=6, n_c=32, C=64, F=256, x="f32", w="f32", act="relu"),
        # odd sizes throughout, 20 chunks of 77 points, 32-bit weights
        dict(name="linear_grad_ragged", kind="linear_grad", N=20, n_c=77, C=1000, F=2003, x="bf16", w="f32",
             act="silu"),
        # gradient of linear_batch in eight chunks (537 MB of chunk gradients)
        dict(name="linear_grad_batch", kind="linear_grad", N=8, n_c=1024, C=2048, F=8192, x="bf16", w="bf16",
             act="gelu"),
        # the same for one matrix alone, in 16 bits
        dict(name="ortho_wide", kind="ortho", batch=1, rows=1024, cols=4096, x="bf16"),
        # the toy vocabulary's matrix, higher than wide: latency alone
        dict(name="muon_tiny", kind="muon", batch=1, rows=257, cols=64, x="f32", nesterov=True),
        # the matrices of twelve equal layers at once
        dict(name="muon_layers", kind="muon", batch=12, rows=768, cols=768, x="f32", nesterov=False),
        # the first matrix of a block
        dict(name="muon_block", kind="muon", batch=1, rows=8192, cols=2048, x="f32", nesterov=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A width: as it falls, or rounded to a multiple of 8 or 64, as most models' are."""
    w = _log(rng, lo, hi)
    m = rng.choice([1, 8, 64])
    return max(lo, w // m * m)


_MOST = 8192 * 2048 * 8192   # products of the largest linear layer
_MOST_G = 8 * 2048 * 8192    # values of its chunk gradients
_MOST_NS = 2048 * 2048 * (3 * 8192 + 2048)   # products of the largest matrix's update, a step


def draw(rng):
    kind = rng.choice(["linear", "linear", "linear_grad", "linear_grad", "ortho", "muon"])
    if kind in ("linear", "linear_grad"):
        x = rng.choice(["f32", "bf16", "bf16"])
        w = rng.choice(["f32", "bf16", "bf16"]) if x == "bf16" else "f32"
        C, F = _width(rng, 64, 8192), _width(rng, 64, 8192)
        act = rng.choice(["none", "relu", "gelu", "gelu_tanh", "silu"])
        if kind == "linear":
            T = _log(rng, 1, max(2, min(8192, _MOST // (C * F))))
            return dict(kind=kind, T=T, C=C, F=F, x=x, w=w, act=act, bias=rng.random() < 0.75,
                        residual=rng.random() < 0.5, keep=rng.random() < 0.5)
        N = min(_log(rng, 1, 32), max(1, _MOST_G // (C * F)))
        n_c = _log(rng, 1, max(2, min(8192 // N, _MOST // (C * F * N))))
        return dict(kind=kind, N=N, n_c=n_c, C=C, F=F, x=x, w=w, act=act)
    a, b = _width(rng, 16, 2048), _width(rng, 16, 8192)
    rows, cols = (a, b) if rng.random() < 0.5 else (b, a)
    one = min(a, b) ** 2 * (3 * max(a, b) + min(a, b))
    batch = _log(rng, 1, max(1, min(16, _MOST_NS // one)))
    if kind == "ortho":
        return dict(kind=kind, batch=batch, rows=rows, cols=cols, x=rng.choice(["f32", "bf16"]))
    return dict(kind=kind, batch=batch, rows=rows, cols=cols, x="f32", nesterov=rng.random() < 0.5)


# ------------------------------------------------------------------------------------ the inputs
def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device=_DEV, dtype=torch.float32)


def _gradient(g, c):
    """Matrices as gradients are: a few strong directions above a floor of many weak ones."""
    b, r, n = c["batch"], c["rows"], c["cols"]
    k = max(1, min(r, n) // 16)
    return _randn(g, b, r, k) @ _randn(g, b, k, n) / math.sqrt(k) + 0.5 * _randn(g, b, r, n)


def prepare(case, seed):
    c = dict(case)
    kind = c["kind"]
    g = torch.Generator(device=_DEV).manual_seed(int(seed) + 1)
    s = dict(case=c)
    xt = _TYPES[c["x"]]
    if kind == "ortho":
        s["u"] = _gradient(g, c).to(xt)
        return s
    if kind == "muon":
        s["points"] = 8192                                       # the gradient is a sum over this many
        s["g"] = _gradient(g, c) * math.sqrt(s["points"])
        s["momentum"] = _gradient(g, c) * (4 / math.sqrt(s["points"]))
        s["w"] = _randn(g, c["batch"], c["rows"], c["cols"]) / math.sqrt(c["cols"])
        s["scale"] = 0.2 * math.sqrt(max(c["rows"], c["cols"]))   # an update's entries as large as any matrix's
        return s
    T = c["T"] if kind == "linear" else c["N"] * c["n_c"]
    C, F = c["C"], c["F"]
    s["x"] = _randn(g, T, C).to(xt)                               # rows out of a layer norm
    s["W"] = (_randn(g, F, C) / math.sqrt(C)).to(_TYPES[c["w"]])
    if kind == "linear":
        s["bias"] = 0.2 * _randn(g, F) if c["bias"] else None
        s["residual"] = (1.5 * _randn(g, T, F)).to(xt) if c["residual"] else None
    else:
        s["z"] = _randn(g, T, F).to(xt) if c["act"] != "none" else None
        s["dy"] = _randn(g, T, F).to(xt)
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
    ws = _workspace(gc)
    if kind == "ortho":
        return {"out": gc.gc_orthogonalize(state["u"], ws=ws)}
    if kind == "muon":
        gc.gc_muon_step(state["w"], state["momentum"], state["g"], _LR, state["points"], mu=_MU,
                        nesterov=c["nesterov"], weight_decay=_DECAY, scale=state["scale"], ws=ws)
        return {"w": state["w"], "momentum": state["momentum"]}
    act = {"none": gc.GC_ACT_NONE, "relu": gc.GC_ACT_RELU, "gelu": gc.GC_ACT_GELU,
           "gelu_tanh": gc.GC_ACT_GELU_TANH, "silu": gc.GC_ACT_SILU}[c["act"]]
    if kind == "linear":
        r = gc.gc_linear(state["x"], state["W"], state["bias"], act, residual=state["residual"], z=c["keep"], ws=ws)
        return {k: r[k] for k in (("y", "z") if c["keep"] else ("y",))}
    r = gc.gc_linear_backward(state["dy"], state["x"], state["W"], c["N"], c["n_c"], z=state["z"], act=act, ws=ws)
    return {k: r[k] for k in ("dx", "G", "Gb")}


# ------------------------------------------------------------------------------------ plain forms
def _act(z, act):
    if act == "relu":
        return z.clamp_min(0)
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z)))
    if act == "silu":
        return z / (1 + torch.exp(-z))
    return z


def _slope(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    if act == "gelu_tanh":
        k = math.sqrt(2 / math.pi)
        t = torch.tanh(k * (z + 0.044715 * z * z * z))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * k * (1 + 3 * 0.044715 * z * z)
    s = 1 / (1 + torch.exp(-z))
    return s * (1 + z * (1 - s))


def _plain_linear(state, c):
    t = state["x"].dtype
    z = state["x"].float() @ state["W"].float().T
    if state["bias"] is not None:
        z = z + state["bias"]
    y = _act(z, c["act"])
    if state["residual"] is not None:
        y = y + state["residual"].float()
    return {"y": y.to(t), "z": z.to(t)} if c["keep"] else {"y": y.to(t)}


def _plain_linear_grad(state, c):
    t = state["x"].dtype
    d = state["dy"].float()
    if c["act"] != "none":
        d = d * _slope(state["z"].float(), c["act"])
    chunks = d.view(c["N"], c["n_c"], c["F"])
    G = torch.bmm(chunks.transpose(1, 2), state["x"].float().view(c["N"], c["n_c"], c["C"]))
    return {"dx": (d @ state["W"].float()).to(t), "G": G.view(c["N"], -1), "Gb": chunks.sum(1)}


def _newton_schulz(u):
    """Five steps X <- (a + b X X^T + c (X X^T)^2) X from u over its norm, on the side that is shorter."""
    a, b, c = _COEFF
    high = u.shape[1] > u.shape[2]
    X = u.transpose(1, 2) if high else u
    X = X / torch.sqrt((X * X).sum((1, 2), keepdim=True)).clamp_min(_EPS)
    X = _steps(X, a, b, c)
    return X.transpose(1, 2) if high else X


def _steps(X, a, b, c):
    for _ in range(5):
        A = X @ X.transpose(1, 2)
        X = a * X + (b * A + c * (A @ A)) @ X
    return X


def _plain_ortho(state, c):
    return {"out": _newton_schulz(state["u"].float()).to(state["u"].dtype)}


def _plain_muon(state, c):
    m, w = state["momentum"], state["w"]
    g = state["g"] / state["points"]
    m.mul_(_MU).add_(g)
    o = _newton_schulz(g + _MU * m if c["nesterov"] else m)
    w.mul_(1 - _LR * _DECAY).sub_(_LR * state["scale"] * o)
    return {"w": w, "momentum": m}


_PLAIN = {"linear": _plain_linear, "linear_grad": _plain_linear_grad, "ortho": _plain_ortho, "muon": _plain_muon}


# ------------------------------------------------------------------------------------ the work
def work(case):
    """Bytes: inputs read once, outputs written once.  Operations: the products; of a symmetric product
    half, so that a step of Newton-Schulz on m x n, m <= n, takes m^2 n + m^3 + 2 m^2 n."""
    c, e = case, _BYTES[case["x"]]
    kind = c["kind"]
    if kind in ("ortho", "muon"):
        m, n = min(c["rows"], c["cols"]), max(c["rows"], c["cols"])
        per = 2 * e if kind == "ortho" else 20   # muon: the gradient in, momentum and matrix in and out
        return {"bytes": c["batch"] * m * n * per, "flops": 5 * c["batch"] * m * m * (3 * n + m)}
    C, F = c["C"], c["F"]
    if kind == "linear":
        T = c["T"]
        outs = 1 + c["residual"] + c["keep"]
        return {"bytes": T * C * e + F * C * _BYTES[c["w"]] + T * F * e * outs + 4 * F * c["bias"],
                "flops": 2 * T * C * F}
    T = c["N"] * c["n_c"]
    rows = T * F * e * (1 if c["act"] == "none" else 2)
    return {"bytes": rows + 2 * T * C * e + F * C * _BYTES[c["w"]] + 4 * c["N"] * F * (C + 1), "flops": 4 * T * C * F}


# ------------------------------------------------------------------------------------ 64 bits
def _sigma(t):
    return torch.special.expit(t)


def exact(case, seed):
    s, c = prepare(case, seed), dict(case)
    kind = c["kind"]
    if kind in ("ortho", "muon"):
        r = {}
        if kind == "ortho":
            u = s["u"].double()
        else:
            g = s["g"].double().div_(s["points"])
            r["momentum"] = torch.lerp(g, s["momentum"].double() + g, _MU)   # g + mu m
            u = torch.add(g, r["momentum"], alpha=_MU) if c["nesterov"] else r["momentum"].clone()
        o = torch.stack([_polynomial(x) for x in u])
        if kind == "ortho":
            return {"out": o}
        r["w"] = s["w"].double() - _LR * (_DECAY * s["w"].double() + s["scale"] * o)
        return r
    x, W = s["x"].double(), s["W"].double()
    if kind == "linear":
        z = torch.einsum("tc,fc->tf", x, W)
        if c["bias"]:
            z += s["bias"].double()
        act = c["act"]
        y = (z if act == "none" else torch.nn.functional.relu(z) if act == "relu"
             else z * torch.special.ndtr(z) if act == "gelu"
             else z * _sigma(2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)) if act == "gelu_tanh"
             else z * _sigma(z))
        if c["residual"]:
            y = y + s["residual"].double()
        return {"y": y, "z": z} if c["keep"] else {"y": y}
    d, act = s["dy"].double(), c["act"]
    if act != "none":
        z = s["z"].double().requires_grad_()
        with torch.enable_grad():
            f = (torch.nn.functional.relu(z) if act == "relu" else z * torch.special.ndtr(z) if act == "gelu"
                 else z * _sigma(2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)) if act == "gelu_tanh"
                 else z * _sigma(z))
            d, = torch.autograd.grad(f, z, d)
    G = torch.stack([torch.einsum("tf,tc->fc", p, q).flatten()
                     for p, q in zip(d.chunk(c["N"]), x.chunk(c["N"]))])
    return {"dx": torch.einsum("tf,fc->tc", d, W), "G": G,
            "Gb": torch.stack([p.sum(0) for p in d.chunk(c["N"])])}


def _polynomial(u):
    """The steps as one matrix Q from the left, Q (u / |u|): all polynomials of u u^T commute."""
    if u.shape[0] > u.shape[1]:
        return _polynomial(u.T).T
    a, b, c = _COEFF
    x = u / max(torch.linalg.matrix_norm(u).item(), _EPS)
    eye = torch.eye(len(x), dtype=x.dtype, device=x.device)
    A, Q = x.mm(x.T), eye
    for _ in range(5):
        P = torch.addmm(b * A + a * eye, A, A, alpha=c)
        Q, A = P.mm(Q), P.mm(A).mm(P)
    return Q.mm(x)
