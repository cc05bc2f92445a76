"""Performance cases of the row normalisation and of activations kept in 8 bits.

Training a deep model over a graph keeps every layer's real-valued input for the backward
pass. These operators normalise the rows of such an input (layer norm), keep the normalised
rows in 8 bits with one power-of-two scale per 32 columns (a checkpoint), and use the
checkpoint in the backward pass: in the norm's own gradient and in the gradient of the weights
of the product that follows it.

* ``norm``         layer norm's forward, rows and their statistics, with or without the 8-bit
                   checkpoint of the normalised rows from the same pass (then read back, as a
                   backward pass that recomputes does).
* ``norm_back``    its backward: the input's gradient and those of gamma and beta, from the
                   layer's input or from the checkpoint.
* ``checkpoint``   any activation to 8 bits and back.
* ``weight_grad``  the gradient of W and of the bias in Z = (gamma v + beta) W + b from the
                   checkpoint v and dZ.

Sizes are those of the graphs and layers that this repository names (Cora, PubMed, Reddit, a
million nodes, 169,343 nodes), and one serving call of a single node.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"
EPS = 1e-5
GROUP = 32
DTYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}
BYTES = {"float32": 4, "bfloat16": 2, "float16": 2}

# The largest listed cases: no drawn case has more elements, or more products.
MAX_NORM = 232965 * 602
MAX_BACK = (1 << 20) * 256
MAX_CHECKPOINT = (1 << 20) * 512
MAX_PRODUCTS = (1 << 20) * 512 * 256


def listed():
    return [
        # The smallest call: one node's row normalised in a serving loop; latency alone.
        dict(name="norm_one", kind="norm", N=1, K=203, dtype="float32", checkpoint=False),
        # First training layers of the citation and the social graph, real features of odd width.
        dict(name="norm_cora", kind="norm", N=2708, K=1433, dtype="float32", checkpoint=True),
        dict(name="norm_reddit", kind="norm", N=232965, K=602, dtype="float32", checkpoint=True),
        # A wide layer in half precision, inference: an odd number of rows.
        dict(name="norm_wide", kind="norm", N=8191, K=8192, dtype="float16", checkpoint=False),
        # Backward from the input itself (no checkpoint kept), in half precision, a small graph.
        dict(name="norm_back_pubmed", kind="norm_back", N=19717, K=500, dtype="float16",
             source="input"),
        # Backward from the checkpoint: the social graph, and a narrow layer on a million nodes.
        dict(name="norm_back_reddit", kind="norm_back", N=232965, K=602, dtype="float32",
             source="checkpoint"),
        dict(name="norm_back_1m", kind="norm_back", N=1 << 20, K=256, dtype="bfloat16",
             source="checkpoint"),
        # An activation put away and taken out again: narrow hidden rows, and a million rows.
        dict(name="checkpoint_170k", kind="checkpoint", N=169343, K=128, dtype="float32"),
        dict(name="checkpoint_1m", kind="checkpoint", N=1 << 20, K=512, dtype="bfloat16"),
        # The weights' gradient behind the norm: few rows of many features (latency), the social
        # graph's first layer with the fp32 gradients that the aggregation returns, and a wide
        # layer on a million nodes with bf16 gradients.
        dict(name="weight_grad_cora", kind="weight_grad", N=2708, K=1433, F=64, dtype="float32"),
        dict(name="weight_grad_reddit", kind="weight_grad", N=232965, K=602, F=128,
             dtype="float32"),
        dict(name="weight_grad_1m", kind="weight_grad", N=1 << 20, K=512, F=256,
             dtype="bfloat16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("norm", "norm_back", "checkpoint", "weight_grad"))
    N, K = _log_int(rng, 1, 1 << 20), _log_int(rng, 32, 8192)
    dtype = rng.choice(("float32", "float32", "bfloat16", "float16"))
    if kind == "norm":
        checkpoint = rng.random() < 0.6
        return dict(kind=kind, N=max(1, min(N, MAX_NORM // K)), K=K, dtype=dtype,
                    checkpoint=checkpoint)
    if kind == "norm_back":
        most = MAX_BACK if dtype != "float32" else MAX_NORM
        return dict(kind=kind, N=max(1, min(N, most // K)), K=K, dtype=dtype,
                    source=rng.choice(("input", "checkpoint")))
    if kind == "checkpoint":
        most = MAX_CHECKPOINT if dtype != "float32" else MAX_CHECKPOINT // 2
        return dict(kind=kind, N=max(1, min(N, most // K)), K=K, dtype=dtype)
    F = _log_int(rng, 4, 256)
    parts = {"float32": 3, "float16": 2, "bfloat16": 1}[dtype]
    N = max(1, min(N, MAX_PRODUCTS // (K * F * parts), MAX_CHECKPOINT // K))
    return dict(kind=kind, N=N, K=K, F=F, dtype=dtype)


def _groups(K):
    return (K + GROUP - 1) // GROUP


# ------------------------------------------------------------------- inputs ----
def _activations(c, g):
    """Rows as a layer in training sees them: every row with its own level and spread, a few
    columns much larger than the rest, rounded to the case's type."""
    N, K = c["N"], c["K"]
    X = torch.randn((N, K), generator=g, device=DEV)
    column = torch.exp(0.5 * torch.randn(K, generator=g, device=DEV))
    X *= column
    X *= torch.exp(0.3 * torch.randn((N, 1), generator=g, device=DEV))
    X += 0.5 * torch.randn((N, 1), generator=g, device=DEV) + 0.2
    return X.to(DTYPES[c["dtype"]])


def _gradients(c, cols, g):
    """Gradients of rows of ``cols`` columns, some rows (labelled nodes) much larger."""
    N = c["N"]
    G = torch.randn((N, cols), generator=g, device=DEV)
    G *= 0.05 * torch.exp(torch.randn((N, 1), generator=g, device=DEV))
    return G.to(DTYPES[c["dtype"]])


def _checkpoint_buffers(N, K):
    """q (N x K int8, rows 16-byte aligned) and exponents (N x groups uint8, rows 4-byte)."""
    q = torch.zeros((N, (K + 15) // 16 * 16), dtype=torch.int8, device=DEV)[:, :K]
    e = torch.zeros((N, (_groups(K) + 3) // 4 * 4), dtype=torch.uint8, device=DEV)
    return q, e[:, :_groups(K)]


def prepare(case, seed):
    c = dict(case)
    g = torch.Generator(device=DEV).manual_seed(seed)
    N, K, kind = c["N"], c["K"], c["kind"]
    dtype = DTYPES[c["dtype"]]
    f32 = torch.float32
    s = dict(c=c)
    s["gamma"] = 1.0 + 0.2 * torch.randn(K, generator=g, device=DEV)
    s["beta"] = 0.1 * torch.randn(K, generator=g, device=DEV)
    empty = lambda *shape, dtype=f32: torch.empty(shape, dtype=dtype, device=DEV)
    if kind in ("norm", "norm_back", "checkpoint"):
        s["X"] = _activations(c, g)
    if kind == "norm":
        s["Y"], s["mean"], s["rstd"] = empty(N, K, dtype=dtype), empty(N), empty(N)
        s["q"] = s["e"] = None
        if c["checkpoint"]:
            s["q"], s["e"] = _checkpoint_buffers(N, K)
            s["values"] = empty(N, K, dtype=torch.bfloat16)
    elif kind == "checkpoint":
        s["q"], s["e"] = _checkpoint_buffers(N, K)
        s["values"] = empty(N, K, dtype=dtype)
    elif kind == "norm_back":
        s["dY"] = _gradients(c, K, g)
        x = s["X"].float()
        s["mean"] = x.mean(1)
        x -= s["mean"][:, None]
        s["rstd"] = 1.0 / torch.sqrt(x.square().mean(1) + EPS)
        if c["source"] == "checkpoint":
            x *= s["rstd"][:, None]
            s["q"], s["e"] = _stored(x)
            del s["X"]
        s["dX"], s["dgamma"], s["dbeta"] = empty(N, K, dtype=dtype), empty(K), empty(K)
    else:
        s["q"], s["e"] = _stored(torch.randn((N, K), generator=g, device=DEV))
        s["dZ"] = _gradients(c, c["F"], g)
        s["dW"], s["db"] = empty(K, c["F"]), empty(c["F"])
    return s


def _stored(v):
    """A checkpoint of fp32 rows in the buffers of a program (inputs of the backward cases)."""
    N, K = v.shape
    q, e = _checkpoint_buffers(N, K)
    qv, ev = _quantise(v)
    q.copy_(qv)
    e.copy_(ev)
    return q, e


# --------------------------------------------------------------- plain forms ----
def _quantise(v):
    """q (int8) and biased exponents (uint8) of fp32 rows: per group of 32 columns the least
    power of two 2^e, e >= -126, by which the largest magnitude rounds to at most 127."""
    N, K = v.shape
    G = _groups(K)
    if G * GROUP != K:
        v = torch.nn.functional.pad(v, (0, G * GROUP - K))
    v = v.reshape(N, G, GROUP)
    mantissa, exponent = torch.frexp(v.abs().amax(2))           # in [1/2, 1), or 0
    e = exponent - 7 + (mantissa * 128 >= 127.5).int()
    e = torch.where(mantissa == 0, -126, e).clamp_min(-126)
    down = ((127 - e) << 23).to(torch.int32).view(torch.float32)   # 2^-e, exact
    q = torch.round(v * down[:, :, None]).reshape(N, G * GROUP)[:, :K]
    return q.to(torch.int8), (e + 127).to(torch.uint8)


def _values(q, e):
    """fp32 values of a checkpoint."""
    N, K = q.shape
    up = (e.to(torch.int32) << 23).view(torch.float32)
    return q.float() * up.repeat_interleave(GROUP, 1)[:, :K]


def _plain(s):
    c = s["c"]
    kind, dtype = c["kind"], DTYPES[c["dtype"]]
    if kind == "norm":
        x = s["X"].float()
        mean = x.mean(1)
        x = x - mean[:, None]
        rstd = 1.0 / torch.sqrt((x * x).mean(1) + EPS)
        xhat = x * rstd[:, None]
        out = dict(y=(xhat * s["gamma"] + s["beta"]).to(dtype), mean=mean, rstd=rstd)
        if c["checkpoint"]:
            out["values"] = _values(*_quantise(xhat)).to(torch.bfloat16)
        return out
    if kind == "norm_back":
        if c["source"] == "checkpoint":
            xhat = _values(s["q"], s["e"])
        else:
            xhat = (s["X"].float() - s["mean"][:, None]) * s["rstd"][:, None]
        dy = s["dY"].float()
        g = dy * s["gamma"]
        dx = g - g.mean(1, keepdim=True) - xhat * (g * xhat).mean(1, keepdim=True)
        return dict(dx=(dx * s["rstd"][:, None]).to(dtype), dgamma=(dy * xhat).sum(0),
                    dbeta=dy.sum(0))
    if kind == "checkpoint":
        return dict(values=_values(*_quantise(s["X"].float())).to(dtype))
    dz = s["dZ"].float()
    db = dz.sum(0)
    dw = _values(s["q"], s["e"]).t() @ dz
    return dict(dw=s["gamma"][:, None] * dw + s["beta"][:, None] * db, db=db)


def run(state):
    if not own:
        return _plain(state)
    from paper_2010_07565_gb300 import binding as B
    s = state
    c = s["c"]
    kind = c["kind"]
    if kind == "norm":
        B.bigcn_layer_norm_forward(s["X"], s["gamma"], s["beta"], EPS, s["Y"], mean=s["mean"],
                                   rstd=s["rstd"], q=s["q"], exps=s["e"])
        out = dict(y=s["Y"], mean=s["mean"], rstd=s["rstd"])
        if c["checkpoint"]:
            B.bigcn_checkpoint_unpack(s["q"], s["e"], s["values"])
            out["values"] = s["values"]
        return out
    if kind == "norm_back":
        if "workspace" not in s:            # sized by the library once, kept by the program
            s["workspace"] = torch.empty(
                B.bigcn_layer_norm_backward_workspace_bytes(c["N"], c["K"]), dtype=torch.uint8,
                device=DEV)
        if c["source"] == "checkpoint":
            B.bigcn_layer_norm_backward(s["dY"], s["gamma"], s["rstd"], s["workspace"],
                                        q=s["q"], exps=s["e"], dX=s["dX"], dgamma=s["dgamma"],
                                        dbeta=s["dbeta"])
        else:
            B.bigcn_layer_norm_backward(s["dY"], s["gamma"], s["rstd"], s["workspace"],
                                        X=s["X"], mean=s["mean"], dX=s["dX"],
                                        dgamma=s["dgamma"], dbeta=s["dbeta"])
        return dict(dx=s["dX"], dgamma=s["dgamma"], dbeta=s["dbeta"])
    if kind == "checkpoint":
        B.bigcn_checkpoint_pack(s["X"], s["q"], s["e"])
        B.bigcn_checkpoint_unpack(s["q"], s["e"], s["values"])
        return dict(values=s["values"])
    if "workspace" not in s:
        s["workspace"] = torch.empty(
            B.bigcn_checkpoint_weight_grad_workspace_bytes(c["N"], c["K"], c["F"]),
            dtype=torch.uint8, device=DEV)
    B.bigcn_checkpoint_weight_grad(s["q"], s["e"], s["dZ"], s["workspace"], s["dW"],
                                   gamma=s["gamma"], beta=s["beta"], db=s["db"])
    return dict(dw=s["dW"], db=s["db"])


# --------------------------------------------------------------------- work ----
def work(case):
    c = case
    N, K, b = c["N"], c["K"], BYTES[c["dtype"]]
    kept = N * K + N * _groups(K)                   # a checkpoint's bytes
    if c["kind"] == "norm":
        extra = 2 * kept + 2 * N * K if c["checkpoint"] else 0    # written, read back, its values
        return {"bytes": 2 * b * N * K + 8 * N + 8 * K + extra, "flops": 8 * N * K}
    if c["kind"] == "norm_back":
        source = kept + 4 * N if c["source"] == "checkpoint" else b * N * K + 8 * N
        return {"bytes": 2 * b * N * K + source + 12 * K, "flops": 12 * N * K}
    if c["kind"] == "checkpoint":
        return {"bytes": 2 * b * N * K + 2 * kept, "flops": 3 * N * K}
    F = c["F"]
    return {"bytes": kept + b * N * F + 4 * K * F + 8 * K + 4 * F, "flops": 2 * N * K * F}


# -------------------------------------------------------------------- exact ----
def _power_of_two(n):
    """2^n in 64 bits by its exponent field: pow() may be an ulp off, which moves ties."""
    return ((n + 1023) << 52).view(torch.float64)


def _kept_values(q, e):
    """A checkpoint's values in 64 bits, from its definition: column k of a row is worth q times
    2 to the power of its group's byte less 127."""
    cols = torch.arange(q.shape[1], device=q.device) // GROUP
    return q.double() * _power_of_two(e.long() - 127)[:, cols]


def exact(case, seed):
    s = prepare(case, seed)
    c = s["c"]
    kind = c["kind"]
    if kind == "norm":
        x = s["X"].double()
        mean = x.sum(1) / c["K"]
        var = (x - mean[:, None]).pow(2).sum(1) / c["K"]
        rstd = (var + EPS).pow(-0.5)
        y = torch.addcmul(s["beta"].double(), (x - mean[:, None]) * rstd[:, None],
                          s["gamma"].double())
        out = dict(y=y, mean=mean, rstd=rstd)
        if c["checkpoint"]:
            # Rounding to 8 bits is a step function of values that are themselves rounded
            # to 32 bits first: near a step the nearest 8-bit value has no single answer.
            out["values"] = None
        return out
    if kind == "norm_back":
        if c["source"] == "checkpoint":
            xhat = _kept_values(s["q"], s["e"])
        else:
            xhat = (s["X"].double() - s["mean"].double()[:, None]) * s["rstd"].double()[:, None]
        dy = s["dY"].double()
        dgamma, dbeta = torch.einsum("ik,ik->k", dy, xhat), dy.sum(0)
        g = dy * s["gamma"].double()
        a = g.sum(1) / c["K"]
        b = torch.einsum("ik,ik->i", g, xhat) / c["K"]
        dx = s["rstd"].double()[:, None] * (g - a[:, None] - b[:, None] * xhat)
        return dict(dx=dx, dgamma=dgamma, dbeta=dbeta)
    if kind == "checkpoint":
        x = s["X"].double()
        out = torch.empty_like(x)
        for k in range(0, c["K"], GROUP):
            v = x[:, k:k + GROUP]
            top = v.abs().amax(1, keepdim=True).clamp_min(2.0 ** -200)
            step = _power_of_two(torch.floor(torch.log2(top)).long() - 7)  # too fine: doubled
            for _ in range(3):
                step = torch.where(torch.round(top / step) > 127, 2 * step, step)
            step = step.clamp_min(2.0 ** -126)
            out[:, k:k + GROUP] = torch.round(v / step) * step
        return dict(values=out)
    dz = s["dZ"].double()
    N, K, F = c["N"], c["K"], c["F"]
    dw = torch.zeros((K, F), dtype=torch.float64, device=DEV)
    db = torch.zeros(F, dtype=torch.float64, device=DEV)
    rows = max(1, (1 << 27) // K)
    for r in range(0, N, rows):
        v = _kept_values(s["q"][r:r + rows], s["e"][r:r + rows])
        v = v * s["gamma"].double() + s["beta"].double()
        dw += v.t() @ dz[r:r + rows]
        db += dz[r:r + rows].sum(0)
    return dict(dw=dw, db=db)
