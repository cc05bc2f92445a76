"""Layer norm forward and backward and the 8-bit checkpoints on the GPU against the 64-bit
reference, within the bounds that norm_reference derives; the checkpoints bit for bit."""
import numpy as np
import pytest
import torch

import norm_reference as R
from paper_2010_07565_gb300 import binding as B

pytestmark = pytest.mark.gpu

DTYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}
EPS = 1e-5


def rng(seed):
    return np.random.Generator(np.random.PCG64(seed))


def rows(N, K, seed, dtype, level=0.7):
    r = rng(seed)
    x = r.standard_normal((N, K)) * np.exp(0.4 * r.standard_normal(K)) + \
        level * r.standard_normal((N, 1))
    return torch.from_numpy(x.astype(np.float32)).to(DTYPES[dtype])


def strided(t, pad, offset, device, fill=float("nan")):
    """t's values on the device in rows ``pad`` elements longer, ``offset`` elements into a
    larger buffer (what lies between is ``fill``)."""
    N, K = t.shape
    buf = torch.full((offset + N * (K + pad) + 64,), fill, dtype=t.dtype, device=device)
    v = buf[offset:offset + N * (K + pad)].view(N, K + pad)[:, :K]
    v.copy_(t)
    return v, buf


def f64(t):
    return t.detach().cpu().double().numpy()


def within(got, ref, bound, what):
    got = f64(got) if isinstance(got, torch.Tensor) else got
    assert got.shape == ref.shape, what
    off = np.abs(got - ref)
    bad = ~(off <= bound)
    if bad.any():
        at = np.unravel_index(np.argmax(np.where(bad, off / np.maximum(bound, 1e-300), 0)), off.shape)
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.size} out of bounds, at {at}: "
                             f"{got[at]} for {ref[at]}, bound {np.broadcast_to(bound, off.shape)[at]}")


def params(K, seed):
    r = rng(seed)
    return (1 + 0.3 * r.standard_normal(K)).astype(np.float32), \
        (0.5 * r.standard_normal(K)).astype(np.float32)


SHAPES = [(1, 1), (3, 2), (1, 33), (2, 7), (5, 31), (33, 32), (17, 64), (300, 65), (1001, 96),
          (7, 100), (129, 128), (64, 203), (501, 256), (37, 500), (2000, 511), (333, 602),
          (19, 1000), (9, 1024), (10, 1026), (5, 1433), (4, 2049), (3, 4096), (6, 5003), (2, 8192),
          (3, 8200), (2, 16385), (2, 33001), (1, 70001)]


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("N,K", SHAPES)
def test_forward(cuda_device, N, K, dtype):
    x = rows(N, K, N + K, dtype)
    gamma, beta = params(K, K)
    X = x.to(cuda_device)
    g, b = torch.from_numpy(gamma).to(cuda_device), torch.from_numpy(beta).to(cuda_device)
    Y, mean, rstd, q, exps = B.layer_norm_forward(X, g, b, EPS)
    ry, rm, rr, rx = R.forward(f64(x), gamma, beta, EPS)
    ey, em, er, ex = R.forward_bounds(f64(x), gamma, beta, EPS, dtype)
    within(Y, ry, ey, "Y")
    within(mean, rm, em, "mean")
    within(rstd, rr, er, "rstd")
    # The checkpoint is of fp32 xhat: half a step and xhat's own error from the reference,
    # in steps that the group's largest magnitude calls for.
    qn, en = q.cpu().numpy(), exps.cpu().numpy()
    step = np.repeat(2.0 ** (en.astype(float) - 127), 32, axis=1)[:, :K]
    within(R.values(qn, en), rx, step / 2 + ex, "checkpoint")
    top = np.stack([np.abs(rx[:, k:k + 32]).max(1) for k in range(0, K, 32)], 1)
    slack = np.stack([ex[:, k:k + 32].max(1) for k in range(0, K, 32)], 1)
    small = 2.0 ** (en.astype(float) - 128)
    assert ((en == 1) | ((top + slack) / small >= 127.5)).all()
    assert np.abs(qn.astype(int)).max() <= 127


@pytest.mark.parametrize("N,K", [(3, 2), (33, 64), (40, 203), (21, 602), (5, 1433), (3, 4096),
                                 (2, 9001), (2, 40000)])
def test_fused_checkpoint_equals_packing_xhat(cuda_device, N, K):
    """Without gamma and beta Y is xhat in fp32: packed by the other call it gives the same
    bytes. Mean, rstd and Y do not depend on whether a checkpoint is written."""
    X = rows(N, K, 5 * N + K, "float32").to(cuda_device)
    Y, mean, rstd, q, exps = B.layer_norm_forward(X, None, None, EPS)
    q2, e2 = B.checkpoint_pack(Y)
    assert torch.equal(q, q2) and torch.equal(exps, e2)
    Y3, mean3, rstd3, _, _ = B.layer_norm_forward(X, None, None, EPS, checkpoint=False)
    assert torch.equal(Y, Y3) and torch.equal(mean, mean3) and torch.equal(rstd, rstd3)


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("pad,offset", [(1, 1), (2, 2), (3, 0), (8, 4), (0, 8), (16, 3)])
@pytest.mark.parametrize("K", [64, 98, 203, 1024])
def test_forward_strides_and_offsets(cuda_device, K, pad, offset, dtype):
    """Rows of other strides and alignments give what aligned ones give, bit for bit but for
    the order of the sums; nothing outside the rows is written."""
    N = 35
    x = rows(N, K, K + pad, dtype)
    gamma, beta = params(K, K)
    X, _ = strided(x, pad, offset, cuda_device)
    Yv, buf = strided(torch.zeros_like(x), pad, offset, cuda_device, fill=7.0)
    g, _ = strided(torch.from_numpy(gamma)[None], 0, offset, cuda_device)
    b, _ = strided(torch.from_numpy(beta)[None], 0, offset, cuda_device)
    mean, rstd = torch.empty(N, device=cuda_device), torch.empty(N, device=cuda_device)
    kq, ke = (K + 15) // 16 * 16, ((K + 31) // 32 + 3) // 4 * 4
    qb = torch.full((N + 1, kq + 32), 99, dtype=torch.int8, device=cuda_device)
    eb = torch.full((N + 1, ke + 8), 99, dtype=torch.uint8, device=cuda_device)
    q, exps = qb[:N, :K], eb[:N, :(K + 31) // 32]
    B.bigcn_layer_norm_forward(X, g[0], b[0], EPS, Yv, mean, rstd, q, exps)
    ry, rm, rr, rx = R.forward(f64(x), gamma, beta, EPS)
    ey, em, er, ex = R.forward_bounds(f64(x), gamma, beta, EPS, dtype)
    within(Yv, ry, ey, "Y")
    within(mean, rm, em, "mean")
    within(rstd, rr, er, "rstd")
    en = exps.cpu().numpy()
    step = np.repeat(2.0 ** (en.astype(float) - 127), 32, axis=1)[:, :K]
    within(R.values(q.cpu().numpy(), en), rx, step / 2 + ex, "checkpoint")
    Yv.fill_(7.0)
    assert (buf == 7.0).all()
    # Padding up to 16 and 4 bytes is 0, beyond it untouched.
    assert (qb[:N, K:kq] == 0).all() and (qb[:N, kq:] == 99).all() and (qb[N] == 99).all()
    assert (eb[:N, (K + 31) // 32:ke] == 0).all() and (eb[:N, ke:] == 99).all()
    assert (eb[N] == 99).all()


@pytest.mark.parametrize("K", [5, 64, 602, 5000])
def test_forward_special_rows(cuda_device, K):
    """Constant rows, rows far from 0, tiny and huge ones; NaN and infinity stay in their row."""
    x = rows(9, K, 3, "float32").numpy()
    x[0] = 4.25
    x[1] = x[1] + 3000.0
    x[2] *= 1e-12
    x[3] *= 1e12
    x[4, K // 2] = np.nan
    x[5, 0] = np.inf
    x[6, K - 1] = -np.inf
    x[7] = 0.0
    Y, mean, rstd, q, exps = B.layer_norm_forward(torch.from_numpy(x).to(cuda_device), None, None,
                                                  EPS)
    fine = [0, 1, 2, 3, 7, 8]
    one, zero = np.ones(K), np.zeros(K)
    ry, rm, rr, rx = R.forward(x[fine], one, zero, EPS)
    ey, em, er, _ = R.forward_bounds(x[fine], one, zero, EPS, "float32")
    within(Y[fine], ry, ey, "Y")
    within(mean[fine], rm, em, "mean")
    within(rstd[fine], rr, er, "rstd")
    bad = [4, 5, 6]
    assert torch.isnan(Y[bad]).all() and (exps[bad] == 255).all()
    assert torch.isnan(B.checkpoint_unpack(q, exps)[bad]).all()
    assert not torch.isnan(B.checkpoint_unpack(q, exps)[fine]).any()
    assert (Y[[0, 7]] == 0).all() and (q[[0, 7]] == 0).all()


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("source", ["input", "checkpoint"])
@pytest.mark.parametrize("N,K", SHAPES)
def test_backward(cuda_device, N, K, source, dtype):
    x = rows(N, K, 2 * N + K, dtype)
    dy = (0.1 * rows(N, K, 7 * N + K, "float32", level=0.2)).to(DTYPES[dtype])
    gamma, beta = params(K, K + 1)
    _, rm, rr, rx = R.forward(f64(x), gamma, beta, EPS)
    mean, rstd = rm.astype(np.float32), rr.astype(np.float32)
    t = lambda a: torch.from_numpy(a).to(cuda_device)
    if source == "input":
        xhat = (f64(x) - mean[:, None].astype(np.float64)) * rstd[:, None].astype(np.float64)
        kw, ex = dict(X=x.to(cuda_device), mean=t(mean)), 2 * R.U * np.abs(xhat)
    else:
        q, exps = B.checkpoint_pack(t(rx.astype(np.float32)))
        xhat, ex = R.values(q.cpu().numpy(), exps.cpu().numpy()), np.zeros((N, K))
        kw = dict(q=q, exps=exps)
    dX, dg, db = B.layer_norm_backward(dy.to(cuda_device), t(gamma), t(rstd), **kw)
    rdx, rdg, rdb = R.backward(f64(dy), gamma, xhat, rstd.astype(np.float64))
    e, eg, eb = R.backward_bounds(f64(dy), gamma, xhat, rstd.astype(np.float64), dtype, ex)
    within(dX, rdx, e, "dX")
    within(dg, rdg, eg, "dgamma")
    within(db, rdb, eb, "dbeta")


@pytest.mark.parametrize("K", [6, 40, 203])
def test_backward_matches_differences(cuda_device, K):
    """dX, dgamma and dbeta against central differences of the 64-bit forward: 1e-4 of their
    scale (the differences' own error, h^2, is 1e-8 of it and the fp32 gradient's 1e-6)."""
    N, h = 4, 1e-4
    r = rng(K)
    x = rows(N, K, K, "float32")
    gamma, beta = params(K, 3)
    dy = r.standard_normal((N, K)).astype(np.float32)
    t = lambda a: torch.from_numpy(a).to(cuda_device)
    X = x.to(cuda_device)
    _, mean, rstd, _, _ = B.layer_norm_forward(X, t(gamma), t(beta), EPS, checkpoint=False)
    dX, dg, db = B.layer_norm_backward(t(dy), t(gamma), rstd, X=X, mean=mean)
    loss = lambda x, g, b: (R.forward(x, g, b, EPS)[0] * dy).sum()
    x64, g64, b64 = f64(x), gamma.astype(np.float64), beta.astype(np.float64)
    for _ in range(6):
        vx, vg, vb = r.standard_normal((N, K)), r.standard_normal(K), r.standard_normal(K)
        d = (loss(x64 + h * vx, g64, b64) - loss(x64 - h * vx, g64, b64)) / (2 * h)
        assert abs(d - (f64(dX) * vx).sum()) <= 1e-4 * (np.abs(f64(dX) * vx).sum() + 1e-3)
        d = (loss(x64, g64 + h * vg, b64) - loss(x64, g64 - h * vg, b64)) / (2 * h)
        assert abs(d - (f64(dg) * vg).sum()) <= 1e-4 * np.abs(f64(dg) * vg).sum()
        d = (loss(x64, g64, b64 + h * vb) - loss(x64, g64, b64 - h * vb)) / (2 * h)
        assert abs(d - (f64(db) * vb).sum()) <= 1e-4 * np.abs(f64(db) * vb).sum()


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("pad,offset", [(1, 1), (2, 2), (8, 0), (5, 3)])
@pytest.mark.parametrize("K", [64, 98, 203, 1024])
def test_backward_strides(cuda_device, K, pad, offset, dtype):
    N = 77
    x = rows(N, K, K, dtype)
    dy = rows(N, K, K + 1, dtype)
    gamma, beta = params(K, K)
    _, rm, rr, _ = R.forward(f64(x), gamma, beta, EPS)
    t = lambda a: torch.from_numpy(a.astype(np.float32)).to(cuda_device)
    X, _ = strided(x, pad, offset, cuda_device)
    dY, _ = strided(dy, pad, offset, cuda_device)
    dX, buf = strided(torch.zeros_like(x), pad, offset, cuda_device, fill=7.0)
    ws = torch.empty(B.bigcn_layer_norm_backward_workspace_bytes(N, K), dtype=torch.uint8,
                     device=cuda_device)
    dg, db = torch.empty(K, device=cuda_device), torch.empty(K, device=cuda_device)
    mean, rstd = t(rm), t(rr)
    B.bigcn_layer_norm_backward(dY, t(gamma), rstd, ws, X=X, mean=mean, dX=dX, dgamma=dg,
                                dbeta=db)
    xhat = (f64(x) - f64(mean)[:, None]) * f64(rstd)[:, None]
    rdx, rdg, rdb = R.backward(f64(dy), gamma, xhat, f64(rstd))
    e, eg, eb = R.backward_bounds(f64(dy), gamma, xhat, f64(rstd), dtype,
                                  2 * R.U * np.abs(xhat))
    within(dX, rdx, e, "dX")
    within(dg, rdg, eg, "dgamma")
    within(db, rdb, eb, "dbeta")
    dX.fill_(7.0)
    assert (buf == 7.0).all()


@pytest.mark.parametrize("N,K", [(1, 203), (700, 602), (3, 9000), (5000, 64)])
def test_backward_parts(cuda_device, N, K):
    """Each output alone is what it is with the others; repeated calls agree bit for bit."""
    dy = rows(N, K, 1, "float32").to(cuda_device)
    gamma = torch.from_numpy(params(K, 2)[0]).to(cuda_device)
    _, _, rstd, q, exps = B.layer_norm_forward(rows(N, K, 3, "float32").to(cuda_device))
    full = B.layer_norm_backward(dy, gamma, rstd, q=q, exps=exps)
    again = B.layer_norm_backward(dy, gamma, rstd, q=q, exps=exps)
    assert all(torch.equal(a, b) for a, b in zip(full, again))
    ws = torch.empty(B.bigcn_layer_norm_backward_workspace_bytes(N, K), dtype=torch.uint8,
                     device=cuda_device)
    for n, name in enumerate(("dX", "dgamma", "dbeta")):
        out = torch.full_like(full[n], float("nan"))
        B.bigcn_layer_norm_backward(dy, gamma, rstd, None if n == 0 else ws, q=q, exps=exps,
                                    **{name: out})
        assert torch.equal(out, full[n]), name
    # gamma = None is gamma = 1.
    one = B.layer_norm_backward(dy, torch.ones_like(gamma), rstd, q=q, exps=exps)
    none = B.layer_norm_backward(dy, None, rstd, q=q, exps=exps)
    assert all(torch.equal(a, b) for a, b in zip(one, none))


def test_backward_no_rows_and_nan_rows(cuda_device):
    K = 70
    e = lambda *s, dtype=torch.float32: torch.empty(s, dtype=dtype, device=cuda_device)
    dg, db = e(K).fill_(3), e(K).fill_(3)
    q, exps = B.checkpoint_buffers(0, K, cuda_device)
    B.bigcn_layer_norm_backward(e(0, K), None, e(0), None, q=q, exps=exps, dX=e(0, K), dgamma=dg,
                                dbeta=db)
    assert (dg == 0).all() and (db == 0).all()
    Y, mean, rstd, _, _ = B.layer_norm_forward(e(0, K))
    assert Y.shape == (0, K)
    X = rows(5, K, 4, "float32").to(cuda_device)
    X[2, 3] = float("nan")
    _, _, rstd, q, exps = B.layer_norm_forward(X)
    dX, dg, db = B.layer_norm_backward(torch.ones_like(X), None, rstd, q=q, exps=exps)
    assert torch.isnan(dX[2]).all() and torch.isfinite(dX[[0, 1, 3, 4]]).all()
    assert torch.isnan(dg).all() and torch.isfinite(db).all()


# ------------------------------------------------------------- checkpoints ----
@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("N,K", [(1, 1), (3, 31), (40, 32), (17, 33), (9, 64), (130, 203),
                                 (5, 602), (64, 128), (3, 1433), (2, 8192), (1, 20001)])
@pytest.mark.parametrize("pad,offset", [(0, 0), (1, 1), (6, 2)])
def test_pack_and_unpack_bit_for_bit(cuda_device, N, K, pad, offset, dtype):
    x = rows(N, K, N * K, dtype)
    x = x * (10.0 ** torch.linspace(-4, 4, N))[:, None].to(x.dtype)
    X, _ = strided(x, pad, offset, cuda_device)
    q, exps = B.checkpoint_pack(X)
    rq, re = R.pack(f64(x))
    assert np.array_equal(q.cpu().numpy(), rq) and np.array_equal(exps.cpu().numpy(), re)
    gamma, beta = params(K, 9)
    v = R.values(rq, re)
    for out in DTYPES:
        got = B.checkpoint_unpack(q, exps, DTYPES[out])
        # bf16 and fp32 hold the values exactly; fp16 rounds those outside its range.
        # (Groups with an fp16 input past its range, an infinity, are NaN.)
        assert np.array_equal(f64(got), f64(torch.from_numpy(v).to(DTYPES[out])), equal_nan=True)
        Xo, buf = strided(torch.zeros(N, K, dtype=DTYPES[out]), pad, offset, cuda_device, fill=7.0)
        B.bigcn_checkpoint_unpack(q, exps, Xo, torch.from_numpy(gamma).to(cuda_device),
                                  torch.from_numpy(beta).to(cuda_device))
        ref = v * gamma + beta
        # One fused multiply-add in fp32, then the rounding to the type.
        r, a = R.OUT_ROUND[out]
        e = R.U * np.abs(ref)
        fine = np.abs(ref) < 60000.0 if out == "float16" else np.isfinite(ref)
        assert np.array_equal(np.isnan(f64(Xo)), np.isnan(ref))
        within(f64(Xo)[fine], ref[fine], (e + r * (np.abs(ref) + e) + a)[fine], "affine")
        Xo.fill_(7.0)
        assert (buf == 7.0).all()


@pytest.mark.parametrize("dtype", list(DTYPES))
def test_pack_special_values(cuda_device, dtype):
    x = torch.zeros((6, 160), dtype=DTYPES[dtype])
    tiny = {"float32": 2.0 ** -149, "bfloat16": 2.0 ** -133, "float16": 2.0 ** -24}[dtype]
    big = torch.finfo(DTYPES[dtype]).max
    x[0, 3], x[0, 40], x[0, 70], x[0, 100] = tiny, float("inf"), float("nan"), -float("inf")
    x[1, 0], x[1, 33], x[1, 65] = big, -big, tiny * 3
    x[2, 0], x[2, 1], x[2, 32], x[2, 64] = 127.5, 0.5, 127.25, -0.0
    x[3, 0:32] = torch.arange(32) * 0.5
    x[4, 0], x[4, 1] = 64.0, 0.5                       # a tie, rounded to even
    q, exps = B.checkpoint_pack(x.to(cuda_device))
    rq, re = R.pack(f64(x))
    finite = re != 255
    assert np.array_equal(exps.cpu().numpy(), re)
    keep = np.repeat(finite, 32, axis=1)[:, :160]
    assert np.array_equal(q.cpu().numpy()[keep], rq[keep])
    back = f64(B.checkpoint_unpack(q, exps))
    assert np.array_equal(np.isnan(back), ~keep)


def test_pack_no_rows_and_other_stream(cuda_device):
    X = torch.empty((0, 50), device=cuda_device)
    q, exps = B.checkpoint_pack(X)
    assert B.checkpoint_unpack(q, exps).shape == (0, 50)
    X = rows(500, 300, 1, "float32").to(cuda_device)
    want = B.checkpoint_pack(X)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = B.checkpoint_buffers(500, 300, cuda_device)
    back = torch.empty_like(X)
    B.bigcn_checkpoint_pack(X, *got, stream=s)
    B.bigcn_checkpoint_unpack(*got, back, stream=s)
    Y = torch.empty_like(X)
    B.bigcn_layer_norm_forward(X, None, None, EPS, Y, stream=s)
    s.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    assert torch.equal(back, B.checkpoint_unpack(*want))
    assert torch.equal(Y, B.layer_norm_forward(X)[0])


def test_offsets_past_32_bits(cuda_device):
    """More than 2^32 elements: the last rows are those of a small call."""
    N, K = 70001, 65544
    X = torch.empty((N, K), dtype=torch.float16, device=cuda_device)
    for r in range(0, N, 4096):
        X[r:r + 4096].normal_()
    q, exps = B.checkpoint_buffers(N, K, cuda_device)
    Y, mean, rstd = torch.empty_like(X), torch.empty(N, device=cuda_device), \
        torch.empty(N, device=cuda_device)
    B.bigcn_layer_norm_forward(X, None, None, EPS, Y, mean, rstd, q, exps)
    part = X[-3:].clone()
    y2, m2, r2, q2, e2 = B.layer_norm_forward(part, None, None, EPS)
    assert torch.equal(Y[-3:], y2) and torch.equal(q[-3:], q2) and torch.equal(exps[-3:], e2)
    dX, dg, _ = B.layer_norm_backward(X, None, rstd, q=q, exps=exps)
    dx2, _, _ = B.layer_norm_backward(part, None, r2, q=q2, exps=e2)
    assert torch.equal(dX[-3:], dx2) and torch.isfinite(dg).all()
    B.bigcn_checkpoint_pack(X, q, exps)
    q3, e3 = B.checkpoint_pack(part)
    assert torch.equal(q[-3:], q3) and torch.equal(exps[-3:], e3)
    B.bigcn_checkpoint_unpack(q, exps, X)
    assert torch.equal(X[-3:], B.checkpoint_unpack(q3, e3, torch.float16))


def test_binding_refusals(cuda_device):
    X = torch.zeros((4, 40), device=cuda_device)
    q, exps = B.checkpoint_buffers(4, 40, cuda_device)
    with pytest.raises(ValueError):
        B.bigcn_checkpoint_pack(X.double(), q, exps)
    with pytest.raises(ValueError):
        B.bigcn_checkpoint_pack(X, q[:3], exps)
    with pytest.raises(ValueError):
        B.bigcn_checkpoint_pack(X, q.view(torch.uint8), exps)
    with pytest.raises(ValueError):
        B.bigcn_layer_norm_forward(X, torch.ones(39, device=cuda_device), None, EPS,
                                   torch.empty_like(X))
    with pytest.raises(ValueError):
        B.bigcn_layer_norm_forward(X, None, None, EPS, torch.empty_like(X).half())
    with pytest.raises(B.BigcnError):
        B.bigcn_layer_norm_forward(X, None, None, -1.0, torch.empty_like(X))
    with pytest.raises(B.BigcnError):
        B.bigcn_layer_norm_forward(X, None, None, EPS, X)
    with pytest.raises(B.BigcnError):
        B.bigcn_checkpoint_pack(X, torch.empty((4, 40), dtype=torch.int8, device=cuda_device), exps)


# Enough rows for the kernels that stage them in shared memory: widths whose rows start at
# every multiple of their element's size, several rows a stage, a last set that is not full,
# matrices that begin and end off 16-byte boundaries.
MANY = [("float32", 20011, 602, 0, 0), ("float32", 39001, 128, 0, 0), ("float32", 10007, 603, 0, 0),
        ("float32", 9999, 1024, 0, 0), ("float32", 10001, 601, 2, 3), ("float32", 5003, 1433, 0, 0),
        ("float32", 12000, 300, 4, 4), ("float32", 9973, 997, 0, 1), ("float32", 20000, 140, 1, 2),
        ("bfloat16", 40007, 256, 0, 0), ("bfloat16", 20001, 601, 0, 0),
        ("bfloat16", 20003, 602, 0, 2), ("bfloat16", 10005, 1000, 4, 4),
        ("bfloat16", 10005, 1021, 3, 7), ("float16", 39999, 260, 0, 0),
        ("float16", 10003, 513, 0, 5), ("float16", 5001, 2050, 0, 0), ("float16", 10111, 770, 2, 6)]


@pytest.mark.parametrize("keep", [False, True])
@pytest.mark.parametrize("dtype,N,K,pad,offset", MANY)
def test_forward_many_rows(cuda_device, dtype, N, K, pad, offset, keep):
    x = rows(N, K, N + K, dtype)
    gamma, beta = params(K, K)
    X, _ = strided(x, pad, offset, cuda_device)
    Yv, buf = strided(torch.zeros_like(x), pad, offset, cuda_device, fill=7.0)
    mean, rstd = torch.empty(N, device=cuda_device), torch.empty(N, device=cuda_device)
    q, exps = B.checkpoint_buffers(N, K, cuda_device) if keep else (None, None)
    t = lambda a: torch.from_numpy(a).to(cuda_device)
    B.bigcn_layer_norm_forward(X, t(gamma), t(beta), EPS, Yv, mean, rstd, q, exps)
    ry, rm, rr, rx = R.forward(f64(x), gamma, beta, EPS)
    ey, em, er, ex = R.forward_bounds(f64(x), gamma, beta, EPS, dtype)
    within(Yv, ry, ey, "Y")
    within(mean, rm, em, "mean")
    within(rstd, rr, er, "rstd")
    if keep:
        en = exps.cpu().numpy()
        step = np.repeat(2.0 ** (en.astype(float) - 127), 32, axis=1)[:, :K]
        within(R.values(q.cpu().numpy(), en), rx, step / 2 + ex, "checkpoint")
        if dtype == "float32":
            B.bigcn_layer_norm_forward(X, None, None, EPS, Yv, None, None, q, exps)
            q2, e2 = B.checkpoint_pack(Yv)
            assert torch.equal(q, q2) and torch.equal(exps, e2)
    Yv.fill_(7.0)
    assert (buf == 7.0).all()
    assert B.device_timeouts() == 0


@pytest.mark.parametrize("source", ["input", "checkpoint"])
@pytest.mark.parametrize("dtype,N,K,pad,offset", MANY)
def test_backward_many_rows(cuda_device, dtype, N, K, pad, offset, source):
    x = rows(N, K, 2 * N + K, dtype)
    dy = (0.1 * rows(N, K, 7 * N + K, "float32", level=0.2)).to(DTYPES[dtype])
    gamma, _ = params(K, K + 1)
    _, rm, rr, rx = R.forward(f64(x), gamma, np.zeros(K), EPS)
    t = lambda a: torch.from_numpy(a.astype(np.float32)).to(cuda_device)
    mean, rstd = t(rm), t(rr)
    if source == "input":
        X, _ = strided(x, pad, offset, cuda_device)
        xhat = (f64(x) - f64(mean)[:, None]) * f64(rstd)[:, None]
        kw, ex = dict(X=X, mean=mean), 2 * R.U * np.abs(xhat)
    else:
        q, exps = B.checkpoint_pack(t(rx))
        xhat, ex = R.values(q.cpu().numpy(), exps.cpu().numpy()), np.zeros((N, K))
        kw = dict(q=q, exps=exps)
    dY, _ = strided(dy, pad, offset, cuda_device)
    dX, buf = strided(torch.zeros_like(dy), pad, offset, cuda_device, fill=7.0)
    ws = torch.empty(B.bigcn_layer_norm_backward_workspace_bytes(N, K), dtype=torch.uint8,
                     device=cuda_device)
    dg, db = torch.empty(K, device=cuda_device), torch.empty(K, device=cuda_device)
    B.bigcn_layer_norm_backward(dY, t(gamma), rstd, ws, dX=dX, dgamma=dg, dbeta=db, **kw)
    rdx, rdg, rdb = R.backward(f64(dy), gamma, xhat, f64(rstd))
    e, eg, eb = R.backward_bounds(f64(dy), gamma, xhat, f64(rstd), dtype, ex)
    within(dX, rdx, e, "dX")
    within(dg, rdg, eg, "dgamma")
    within(db, rdb, eb, "dbeta")
    again = [torch.empty_like(dg), torch.empty_like(db)]
    B.bigcn_layer_norm_backward(dY, t(gamma), rstd, ws, dgamma=again[0], dbeta=again[1], **kw)
    assert torch.equal(again[0], dg) and torch.equal(again[1], db)
    dX.fill_(7.0)
    assert (buf == 7.0).all()
    assert B.device_timeouts() == 0


def test_many_rows_with_nan_and_infinite_rows(cuda_device):
    N, K = 20000, 602
    x = rows(N, K, 5, "float32")
    x[11, 600], x[12, 0], x[N - 1, K - 1] = float("nan"), float("inf"), float("nan")
    bad = torch.zeros(N, dtype=torch.bool)
    bad[[11, 12, N - 1]] = True
    X = x.to(cuda_device)
    Y, mean, rstd, q, exps = B.layer_norm_forward(X)
    assert torch.equal(torch.isnan(Y).all(1).cpu(), bad) and torch.equal(torch.isnan(Y).any(1).cpu(), bad)
    assert torch.equal((exps == 255).all(1).cpu(), bad)
    dX, dg, db = B.layer_norm_backward(torch.ones_like(X), None, rstd, q=q, exps=exps)
    assert torch.equal(torch.isnan(dX).any(1).cpu(), bad)
    assert torch.isnan(dg).all() and torch.isfinite(db).all()
