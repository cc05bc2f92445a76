"""Performance cases of a deep residual layer's operators in training and serving.

A deep model over a graph keeps a stream of rows that every layer adds to. A layer normalises the
rows of that stream, multiplies them by its weights and aggregates; in low precision the product
takes both operands in 4 bits, and in training the gradients of all layers together are clipped.

* ``rms``          the residual's addition and root-mean-square norm of the sum, with or without
                   the normalised rows in 8 bits (a checkpoint, which the backward pass and the
                   weights' gradient read), its values read back as a backward pass does.
* ``rms_back``     its backward: the stream's gradient, with what comes past the layer added, and
                   gamma's, from the forward's sum or from the checkpoint.
* ``fp4``          rows to 4 bits (e2m1) with a power-of-two scale per 32 columns, and back.
* ``fp4_columns``  the same of a weight matrix's columns, which become rows.
* ``fp4_gemm``     the product of two such matrices and a bias.
* ``clip``         the norm of all gradients together, and the gradients scaled down to a limit.

Sizes are those of the graphs and layers that this repository names (Cora, PubMed, Reddit, a
million nodes; up to 8192 features, 256 columns), wider layers of the same kind, and one serving
call of a single node.
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
MAX_RMS = 232965 * 602
MAX_BACK = (1 << 20) * 256
MAX_ROWS = 232965 * 602
MAX_COLUMNS = 8192 * 1024
MAX_GEMM_IN = (1 << 17) * 8192
MAX_GEMM_OUT = 232965 * 602
MAX_PRODUCTS = (1 << 17) * 8192 * 256
MAX_GRADS = 48 * 4096 * 1024


def listed():
    return [
        # The smallest call: one node's row in a serving loop, added and normalised; latency alone.
        dict(name="rms_one", kind="rms", N=1, K=203, dtype="bfloat16", residual=True,
             checkpoint=False),
        # A layer in training on the social graph: sum, norm and the checkpoint for the backward.
        dict(name="rms_reddit", kind="rms", N=232965, K=602, dtype="float32", residual=True,
             checkpoint=True),
        # Backward from the stream itself (no checkpoint kept), in half precision, a small graph.
        dict(name="rms_back_pubmed", kind="rms_back", N=19717, K=500, dtype="float16",
             source="input", past=True),
        # Backward from the checkpoint: a hidden layer on a million nodes.
        dict(name="rms_back_1m", kind="rms_back", N=1 << 20, K=256, dtype="bfloat16",
             source="checkpoint", past=True),
        # Features of the social graph to 4 bits, once per pass of a layer whose input is fp32.
        dict(name="fp4_reddit", kind="fp4", N=232965, K=602, dtype="float32"),
        # The weights of a wide layer, after every update of theirs.
        dict(name="fp4_columns_wide", kind="fp4_columns", K=8192, F=1024, dtype="float32"),
        # One node of the citation graph through its first layer; latency alone.
        dict(name="fp4_gemm_one", kind="fp4_gemm", N=1, K=1433, F=64, dtype="float32", bias=True),
        # The social graph's first layer, forward: fp32 for the aggregation behind it.
        dict(name="fp4_gemm_reddit", kind="fp4_gemm", N=232965, K=602, F=128, dtype="float32",
             bias=True),
        # Its input's gradient: few columns of gradients times the weights' rows, a wide output.
        dict(name="fp4_gemm_back", kind="fp4_gemm", N=232965, K=128, F=602, dtype="float32",
             bias=False),
        # A wide layer's forward pass, half precision behind it.
        dict(name="fp4_gemm_wide", kind="fp4_gemm", N=1 << 17, K=8192, F=256, dtype="bfloat16",
             bias=True),
        # All gradients of the citation graph's two-layer model; latency alone.
        dict(name="clip_cora", kind="clip", layers=2, K=1433, F=64, dtype="float32"),
        # A deep stack of wide layers, matrices in bf16 and vectors in fp32.
        dict(name="clip_stack", kind="clip", layers=48, K=4096, F=1024, dtype="mixed"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("rms", "rms_back", "fp4", "fp4_columns", "fp4_gemm", "fp4_gemm", "clip"))
    N, K = _log_int(rng, 1, 1 << 20), _log_int(rng, 32, 8192)
    F = _log_int(rng, 4, 1024)
    dtype = rng.choice(("float32", "float32", "bfloat16", "float16"))
    if kind == "rms":
        return dict(kind=kind, N=max(1, min(N, MAX_RMS // K)), K=K, dtype=dtype,
                    residual=rng.random() < 0.8, checkpoint=rng.random() < 0.6)
    if kind == "rms_back":
        most = MAX_BACK if dtype != "float32" else MAX_RMS
        return dict(kind=kind, N=max(1, min(N, most // K)), K=K, dtype=dtype,
                    source=rng.choice(("input", "checkpoint")), past=rng.random() < 0.7)
    if kind == "fp4":
        return dict(kind=kind, N=max(1, min(N, MAX_ROWS // K)), K=K, dtype=dtype)
    if kind == "fp4_columns":
        return dict(kind=kind, K=K, F=max(1, min(F, MAX_COLUMNS // K)), dtype=dtype)
    if kind == "fp4_gemm":
        most = min(MAX_GEMM_IN // K, MAX_GEMM_OUT // F, MAX_PRODUCTS // (K * F))
        return dict(kind=kind, N=max(1, min(N, most)), K=K, F=F, dtype=dtype,
                    bias=rng.random() < 0.6)
    layers = _log_int(rng, 1, 100)
    return dict(kind=kind, layers=max(1, min(layers, MAX_GRADS // (K * F))), K=K, F=F,
                dtype=rng.choice(("float32", "mixed", "bfloat16")))


def _groups(K):
    return (K + GROUP - 1) // GROUP


# ------------------------------------------------------------------- inputs ----
def _activations(N, K, dtype, g):
    """Rows as a layer in training sees them: every row with its own level and spread, a few
    columns much larger than the rest, rounded to the case's type."""
    X = torch.randn((N, K), generator=g, device=DEV)
    X *= torch.exp(0.5 * torch.randn(K, generator=g, device=DEV))
    X *= torch.exp(0.3 * torch.randn((N, 1), generator=g, device=DEV))
    X += 0.2 * torch.randn((N, 1), generator=g, device=DEV)
    return X.to(DTYPES[dtype])


def _gradients(N, K, dtype, g):
    """Gradients of rows, some rows (labelled nodes) much larger."""
    G = torch.randn((N, K), generator=g, device=DEV)
    G *= 0.05 * torch.exp(torch.randn((N, 1), generator=g, device=DEV))
    return G.to(DTYPES[dtype])


def _checkpoint_buffers(N, K):
    """q (N x K int8, rows 16-byte aligned) and exponents (N x groups uint8, rows 4-byte)."""
    q = torch.zeros((N, (K + 15) // 16 * 16), dtype=torch.int8, device=DEV)[:, :K]
    e = torch.zeros((N, (_groups(K) + 3) // 4 * 4), dtype=torch.uint8, device=DEV)
    return q, e[:, :_groups(K)]


def _fp4_buffers(N, K):
    """Rows of 4-bit codes, two to a byte (rows 16-byte aligned), and exponents (rows 4-byte)."""
    q = torch.zeros((N, _groups(K) * (GROUP // 2)), dtype=torch.uint8, device=DEV)
    e = torch.zeros((N, (_groups(K) + 3) // 4 * 4), dtype=torch.uint8, device=DEV)
    return q[:, :(K + 1) // 2], e[:, :_groups(K)]


def _grad_shapes(c):
    """Each layer's weights, bias and gamma."""
    K, F = c["K"], c["F"]
    matrix = torch.float32 if c["dtype"] == "float32" else torch.bfloat16
    vector = torch.bfloat16 if c["dtype"] == "bfloat16" else torch.float32
    return [(matrix, K * F), (vector, F), (vector, K)] * c["layers"]


def _views(shapes):
    """({type: one buffer}, its tensors): each starts at a multiple of 64 elements, as allocations
    of their own do at least; the rest is 0."""
    ends, at = {}, []
    for t, n in shapes:
        start = ends.get(t, 0)
        at.append((t, start, n))
        ends[t] = start + (n + 63) // 64 * 64
    flat = {t: torch.zeros(n, dtype=t, device=DEV) for t, n in ends.items()}
    return flat, [flat[t][a:a + n] for t, a, n in at]


def prepare(case, seed):
    c = dict(case)
    g = torch.Generator(device=DEV).manual_seed(seed)
    kind = c["kind"]
    f32 = torch.float32
    s = dict(c=c)
    empty = lambda *shape, dtype=f32: torch.empty(shape, dtype=dtype, device=DEV)
    if kind == "clip":
        shapes = _grad_shapes(c)
        s["flat"], s["grads"] = _views(shapes)
        s["flat_out"], s["out"] = _views(shapes)
        level = torch.exp(torch.randn(len(shapes), generator=g, device=DEV))
        for i, t in enumerate(s["grads"]):
            t.copy_(torch.randn(t.numel(), generator=g, device=DEV) * level[i] * 0.01)
        s["norm"] = empty(1)
        s["max_norm"] = 1.0
        return s
    K, dtype = c["K"], DTYPES[c["dtype"]]
    if kind in ("rms", "rms_back"):
        N = c["N"]
        s["gamma"] = 1.0 + 0.2 * torch.randn(K, generator=g, device=DEV)
        s["X"] = _activations(N, K, c["dtype"], g)
    if kind == "rms":
        s["R"] = _activations(N, K, c["dtype"], g) if c["residual"] else None
        s["S"] = empty(N, K, dtype=dtype) if c["residual"] else None
        s["Y"], s["rstd"] = empty(N, K, dtype=dtype), empty(N)
        s["q"] = s["e"] = None
        if c["checkpoint"]:
            s["q"], s["e"] = _checkpoint_buffers(N, K)
            s["values"] = empty(N, K, dtype=torch.bfloat16)
    elif kind == "rms_back":
        s["dY"] = _gradients(N, K, c["dtype"], g)
        s["dS"] = _gradients(N, K, c["dtype"], g) if c["past"] else None
        x = s["X"].float()
        s["rstd"] = 1.0 / torch.sqrt((x * x).mean(1) + EPS)
        if c["source"] == "checkpoint":
            x *= s["rstd"][:, None]
            s["q"], s["e"] = _checkpoint_buffers(N, K)
            for a, b in zip((s["q"], s["e"]), _to_8_bits(x)):
                a.copy_(b)
            del s["X"]
        s["dX"], s["dgamma"] = empty(N, K, dtype=dtype), empty(K)
    elif kind == "fp4":
        s["X"] = _activations(c["N"], K, c["dtype"], g)
        s["q"], s["e"] = _fp4_buffers(c["N"], K)
        s["values"] = empty(c["N"], K, dtype=torch.bfloat16)
    elif kind == "fp4_columns":
        W = torch.randn((K, c["F"]), generator=g, device=DEV) / math.sqrt(K)
        W *= torch.exp(0.5 * torch.randn((K, 1), generator=g, device=DEV))
        s["W"] = W.to(dtype)
        s["q"], s["e"] = _fp4_buffers(c["F"], K)
        s["values"] = empty(c["F"], K, dtype=torch.bfloat16)
    else:
        N, F = c["N"], c["F"]
        s["a"], s["ae"] = _kept_4_bits(_activations(N, K, "float32", g))
        s["b"], s["be"] = _kept_4_bits(torch.randn((F, K), generator=g, device=DEV) / math.sqrt(K))
        s["bias"] = 0.1 * torch.randn(F, generator=g, device=DEV) if c["bias"] else None
        s["Z"] = empty(N, F, dtype=dtype)
    return s


def _kept_4_bits(v):
    """Rows in 4 bits, in the buffers of a program (operands of the product)."""
    N, K = v.shape
    q, e = _fp4_buffers(N, K)
    code, ev = _to_4_bits(v)
    code = torch.nn.functional.pad(code, (0, K % 2))
    q.copy_(code[:, 0::2] | (code[:, 1::2] << 4))
    e.copy_(ev)
    return q, e


# --------------------------------------------------------------- plain forms ----
def _grouped(v):
    """fp32 rows as N x groups x 32, zeros behind them."""
    N, K = v.shape
    G = _groups(K)
    if G * GROUP != K:
        v = torch.nn.functional.pad(v, (0, G * GROUP - K))
    return v.reshape(N, G, GROUP)


def _power(e):
    """2^e for whole e in [-126, 127], exact."""
    return ((e + 127) << 23).to(torch.int32).view(torch.float32)


def _to_8_bits(v):
    """q (int8) and biased exponents (uint8) of fp32 rows: per group of 32 columns the least
    power of two 2^e, e >= -126, by which the largest magnitude rounds to at most 127."""
    N, K = v.shape
    v = _grouped(v)
    mantissa, exponent = torch.frexp(v.abs().amax(2))           # in [1/2, 1), or 0
    e = exponent - 7 + (mantissa * 128 >= 127.5).int()
    e = torch.where(mantissa == 0, -126, e).clamp_min(-126)
    q = torch.round(v * _power(-e)[:, :, None]).reshape(N, -1)[:, :K]
    return q.to(torch.int8), (e + 127).to(torch.uint8)


def _from_8_bits(q, e):
    K = q.shape[1]
    return q.float() * _power(e.to(torch.int32) - 127).repeat_interleave(GROUP, 1)[:, :K]


def _to_4_bits(v):
    """Codes (uint8, the sign in bit 3) and biased exponents (uint8) of fp32 rows: per group of 32
    columns the least power of two 2^e, e >= -126, by which the largest magnitude rounds to at most
    6; magnitudes 0, 1/2, 1, 3/2, 2, 3, 4, 6, rounded to nearest, ties to the even code."""
    N, K = v.shape
    v = _grouped(v)
    mantissa, exponent = torch.frexp(v.abs().amax(2))
    e = exponent - 3 + (mantissa >= 0.875).int()
    e = torch.where(mantissa == 0, -126, e).clamp_min(-126)
    m = v.abs() * _power(-e)[:, :, None]
    code = ((m > 0.25).to(torch.uint8) + (m >= 0.75) + (m > 1.25) + (m >= 1.75) + (m > 2.5) +
            (m >= 3.5) + (m > 5.0))
    code = (code | ((v < 0).to(torch.uint8) << 3)).reshape(N, -1)[:, :K]
    return code, (e + 127).to(torch.uint8)


def _from_4_bits(code, e):
    """fp32 values of codes and biased exponents."""
    K = code.shape[1]
    m = (code & 7).int()
    low = (m < 2).float() * m.float() * 0.5
    high = (m >= 2).float() * (1.0 + 0.5 * (m & 1).float()) * _power((m >> 1) - 1)
    sign = 1.0 - 2.0 * (code >> 3).float()
    return sign * (low + high) * _power(e.to(torch.int32) - 127).repeat_interleave(GROUP, 1)[:, :K]


def _codes(q, K):
    """The codes of packed bytes: the even column in the low half."""
    return torch.stack((q & 15, q >> 4), 2).reshape(q.shape[0], -1)[:, :K]


def _plain(s):
    c = s["c"]
    kind = c["kind"]
    if kind == "clip":
        norm = torch.sqrt(sum(t.double().square().sum() for t in s["grads"]))
        norm32 = norm.float()
        over = torch.isfinite(norm32) & (norm32 > s["max_norm"])
        factor = torch.where(over, s["max_norm"] / norm, 1.0).float()
        [o.copy_(t.float() * factor) for t, o in zip(s["grads"], s["out"])]
        return dict(norm=norm32.reshape(1), out=[s["flat_out"][t] for t in s["flat_out"]])
    dtype = DTYPES[c["dtype"]]
    if kind == "rms":
        out = {}
        x = s["X"].float()
        if c["residual"]:
            total = (x + s["R"].float()).to(dtype)
            out["sum"] = total
            x = total.float()
        rstd = 1.0 / torch.sqrt((x * x).mean(1) + EPS)
        xhat = x * rstd[:, None]
        out.update(y=(xhat * s["gamma"]).to(dtype), rstd=rstd)
        if c["checkpoint"]:
            out["values"] = _from_8_bits(*_to_8_bits(xhat)).to(torch.bfloat16)
        return out
    if kind == "rms_back":
        if c["source"] == "checkpoint":
            xhat = _from_8_bits(s["q"], s["e"])
        else:
            xhat = s["X"].float() * s["rstd"][:, None]
        dy = s["dY"].float()
        g = dy * s["gamma"]
        dx = (g - xhat * (g * xhat).mean(1, keepdim=True)) * s["rstd"][:, None]
        if c["past"]:
            dx = dx + s["dS"].float()
        return dict(dx=dx.to(dtype), dgamma=(dy * xhat).sum(0))
    if kind == "fp4":
        return dict(values=_from_4_bits(*_to_4_bits(s["X"].float())).to(torch.bfloat16))
    if kind == "fp4_columns":
        columns = s["W"].float().t().contiguous()
        return dict(values=_from_4_bits(*_to_4_bits(columns)).to(torch.bfloat16))
    K = c["K"]
    z = _from_4_bits(_codes(s["a"], K), s["ae"]) @ _from_4_bits(_codes(s["b"], K), s["be"]).t()
    if c["bias"]:
        z = z + s["bias"]
    return dict(z=z.to(dtype))


def run(state):
    if not own:
        return _plain(state)
    from paper_2010_07565_gb300 import binding as B
    s = state
    c = s["c"]
    kind = c["kind"]
    if kind == "clip":
        if "list" not in s:                 # built once by the program that keeps the gradients
            s["list"], s["out_list"] = B.TensorList(s["grads"]), B.TensorList(s["out"])
            s["workspace"] = torch.empty(B.bigcn_grad_norm_workspace_bytes(s["list"]),
                                         dtype=torch.uint8, device=DEV)
        B.bigcn_clip_grad_norm(s["list"], s["max_norm"], s["norm"], s["workspace"],
                               out=s["out_list"])
        return dict(norm=s["norm"], out=[s["flat_out"][t] for t in s["flat_out"]])
    if kind == "rms":
        B.bigcn_rms_norm_forward(s["X"], s["gamma"], EPS, R=s["R"], S=s["S"], Y=s["Y"],
                                 rstd=s["rstd"], q=s["q"], exps=s["e"])
        out = dict(y=s["Y"], rstd=s["rstd"])
        if c["residual"]:
            out["sum"] = s["S"]
        if c["checkpoint"]:
            B.bigcn_checkpoint_unpack(s["q"], s["e"], s["values"])
            out["values"] = s["values"]
        return out
    if kind == "rms_back":
        if "workspace" not in s:            # sized by the library once, kept by the program
            s["workspace"] = torch.empty(
                B.bigcn_rms_norm_backward_workspace_bytes(c["N"], c["K"]), dtype=torch.uint8,
                device=DEV)
        if c["source"] == "checkpoint":
            B.bigcn_rms_norm_backward(s["dY"], s["gamma"], s["rstd"], s["workspace"], q=s["q"],
                                      exps=s["e"], dS=s["dS"], dX=s["dX"], dgamma=s["dgamma"])
        else:
            B.bigcn_rms_norm_backward(s["dY"], s["gamma"], s["rstd"], s["workspace"], S=s["X"],
                                      dS=s["dS"], dX=s["dX"], dgamma=s["dgamma"])
        return dict(dx=s["dX"], dgamma=s["dgamma"])
    if kind == "fp4":
        B.bigcn_fp4_pack(s["X"], s["q"], s["e"])
        B.bigcn_fp4_unpack(s["q"], s["e"], s["values"])
        return dict(values=s["values"])
    if kind == "fp4_columns":
        B.bigcn_fp4_pack_columns(s["W"], s["q"], s["e"])
        B.bigcn_fp4_unpack(s["q"], s["e"], s["values"])
        return dict(values=s["values"])
    B.bigcn_fp4_gemm(s["a"], s["ae"], s["b"], s["be"], c["K"], s["Z"], bias=s["bias"])
    return dict(z=s["Z"])


# --------------------------------------------------------------------- work ----
def work(case):
    c = case
    kind = c["kind"]
    if kind == "clip":
        sizes = [(4 if t == torch.float32 else 2, n) for t, n in _grad_shapes(c)]
        return {"bytes": 2 * sum(b * n for b, n in sizes) + 4, "flops": 3 * sum(n for _, n in sizes)}
    K, b = c["K"], BYTES[c["dtype"]]
    if kind == "rms":
        N = c["N"]
        kept = N * K + N * _groups(K)                   # a checkpoint's bytes
        extra = 2 * kept + 2 * N * K if c["checkpoint"] else 0    # written, read back, its values
        streams = 4 if c["residual"] else 2
        return {"bytes": streams * b * N * K + 4 * N + 4 * K + extra, "flops": 6 * N * K}
    if kind == "rms_back":
        N = c["N"]
        source = N * K + N * _groups(K) if c["source"] == "checkpoint" else b * N * K
        return {"bytes": (3 if c["past"] else 2) * b * N * K + source + 4 * N + 8 * K,
                "flops": 10 * N * K}
    four = lambda rows: rows * ((K + 1) // 2 + _groups(K))
    if kind in ("fp4", "fp4_columns"):
        rows = c["N"] if kind == "fp4" else c["F"]
        return {"bytes": b * rows * K + 2 * four(rows) + 2 * rows * K, "flops": 3 * rows * K}
    N, F = c["N"], c["F"]
    return {"bytes": four(N) + four(F) + b * N * F + (4 * F if c["bias"] else 0),
            "flops": 2 * N * K * F}


# -------------------------------------------------------------------- exact ----
def _power_of_two(n):
    """2^n in 64 bits by its exponent field: pow() may be an ulp off, which moves ties."""
    return ((n + 1023) << 52).view(torch.float64)


def _scales(e, K):
    """Each column's scale in 64 bits: 2 to the power of its group's byte less 127."""
    cols = torch.arange(K, device=e.device) // GROUP
    return _power_of_two(e.long() - 127)[:, cols]


_E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _values_of_4_bits(q, e, K):
    """Packed 4-bit rows in 64 bits, from the definition: a table of the eight magnitudes."""
    table = torch.tensor(_E2M1 + tuple(-v for v in _E2M1), dtype=torch.float64, device=q.device)
    v = torch.empty((q.shape[0], q.shape[1] * 2), dtype=torch.float64, device=q.device)
    v[:, 0::2] = table[(q % 16).long()]
    v[:, 1::2] = table[(q // 16).long()]
    return v[:, :K] * _scales(e, K)


def _nearest_4_bits(x):
    """Rows rounded to 4 bits in 64 bits: the scale by trial, then the nearest of the magnitudes,
    the even code where two are as near."""
    grid = torch.tensor(_E2M1, dtype=torch.float64, device=x.device)
    out = torch.empty_like(x)
    for k in range(0, x.shape[1], GROUP):
        v = x[:, k:k + GROUP]
        top = v.abs().amax(1, keepdim=True)
        n = torch.floor(torch.log2(top.clamp_min(2.0 ** -200))).long() - 4
        for _ in range(4):                              # until what rounds above 6 does not
            n = torch.where(top / _power_of_two(n) >= 7.0, n + 1, n)
        step = _power_of_two(n.clamp_min(-126))
        m = v.abs() / step
        i = torch.bucketize(m, grid, right=True).sub_(1).clamp_(0, 7)      # grid[i] <= m
        j = (i + 1).clamp_max(7)
        below, above = m - grid[i], grid[j] - m
        up = (above < below) | ((above == below) & (i % 2 == 1))
        out[:, k:k + GROUP] = torch.where(up, grid[j], grid[i]) * torch.sign(v) * step
    return out


def exact(case, seed):
    s = prepare(case, seed)
    c = s["c"]
    kind = c["kind"]
    if kind == "clip":
        norm = math.sqrt(sum(float(torch.dot(t.double(), t.double())) for t in s["grads"]))
        factor = min(1.0, s["max_norm"] / norm) if norm > 0.0 else 1.0
        return dict(norm=torch.tensor([norm], dtype=torch.float64),
                    out=[f.double() * factor for f in s["flat"].values()])
    K = c["K"]
    if kind == "rms":
        x = s["X"].double()
        out = {}
        if c["residual"]:
            out["sum"] = x + s["R"].double()
            # The stream holds the sum in its own type, and that is what is normalised.
            x = out["sum"].to(torch.float32).to(DTYPES[c["dtype"]]).double()
        rstd = (x.pow(2).sum(1) / K + EPS).pow(-0.5)
        out["y"] = x * rstd[:, None] * s["gamma"].double()
        out["rstd"] = rstd
        if c["checkpoint"]:
            # Rounding to 8 bits is a step function of values that are themselves rounded
            # to 32 bits first: near a step the nearest 8-bit value has no single answer.
            out["values"] = None
        return out
    if kind == "rms_back":
        if c["source"] == "checkpoint":
            xhat = s["q"].double() * _scales(s["e"], K)
        else:
            xhat = s["X"].double() * s["rstd"].double()[:, None]
        dy = s["dY"].double()
        dgamma = torch.einsum("ik,ik->k", dy, xhat)
        g = dy * s["gamma"].double()
        b = torch.einsum("ik,ik->i", g, xhat) / K
        dx = s["rstd"].double()[:, None] * (g - b[:, None] * xhat)
        if c["past"]:
            dx = dx + s["dS"].double()
        return dict(dx=dx, dgamma=dgamma)
    if kind == "fp4":
        rows = max(1, (1 << 26) // K)
        return dict(values=torch.cat([_nearest_4_bits(s["X"][r:r + rows].double())
                                      for r in range(0, c["N"], rows)]))
    if kind == "fp4_columns":
        return dict(values=_nearest_4_bits(s["W"].double().t().contiguous()))
    N, F = c["N"], c["F"]
    b = _values_of_4_bits(s["b"], s["be"], K).t()
    z = torch.empty((N, F), dtype=torch.float64, device=DEV)
    rows = max(1, (1 << 27) // K)
    for r in range(0, N, rows):
        z[r:r + rows] = _values_of_4_bits(s["a"][r:r + rows], s["ae"][r:r + rows], K) @ b
    if c["bias"]:
        z += s["bias"].double()
    return dict(z=z)
