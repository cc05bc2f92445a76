"""The residual's addition with root-mean-square norm, and its backward, on the GPU against the 64-bit
reference, within the bounds that residual_reference derives."""
import numpy as np
import pytest
import torch

import norm_reference as N_
import residual_reference as R
from paper_2010_07565_gb300 import binding as B
from test_gpu_norm import DTYPES, SHAPES, f64, params, rows, strided, within

pytestmark = pytest.mark.gpu

EPS = 1e-5


def summed(x, r):
    """The stream's rows: the addends' fp32 sum rounded to their type."""
    return (x.float() + r.float()).to(x.dtype)


def check_checkpoint(q, exps, shat, ex, K):
    qn, en = q.cpu().numpy(), exps.cpu().numpy()
    step = np.repeat(2.0 ** (en.astype(float) - 127), 32, axis=1)[:, :K]
    within(N_.values(qn, en), shat, step / 2 + ex, "checkpoint")
    assert np.abs(qn.astype(int)).max(initial=0) <= 127


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("N,K", SHAPES)
def test_forward(cuda_device, N, K, residual, dtype):
    x, r = rows(N, K, N + K, dtype), rows(N, K, N + K + 1, dtype)
    gamma = params(K, K)[0]
    s = summed(x, r) if residual else x
    g = torch.from_numpy(gamma).to(cuda_device)
    Y, S, rstd, q, exps = B.rms_norm_forward(x.to(cuda_device), g, EPS,
                                             R=r.to(cuda_device) if residual else None)
    assert torch.equal(S.cpu(), s)
    ry, rr, rx = R.rms_forward(f64(s), gamma, EPS)
    ey, er, ex = R.rms_forward_bounds(f64(s), gamma, EPS, dtype)
    within(Y, ry, ey, "Y")
    within(rstd, rr, er, "rstd")
    check_checkpoint(q, exps, rx, ex, K)


@pytest.mark.parametrize("N,K", [(3, 2), (33, 64), (40, 203), (21, 602), (5, 1433), (3, 4096),
                                 (2, 9001), (2, 40000)])
def test_outputs_do_not_depend_on_each_other(cuda_device, N, K):
    """Without gamma Y is shat in fp32: packed by the checkpoint's own call it gives the same bytes.
    Each output alone is what it is with the others, in place of an addend too."""
    x, r = (rows(N, K, 5 * N + K + i, "float32").to(cuda_device) for i in (0, 1))
    Y, S, rstd, q, exps = B.rms_norm_forward(x, None, EPS, R=r)
    q2, e2 = B.checkpoint_pack(Y)
    assert torch.equal(q, q2) and torch.equal(exps, e2)
    only = torch.full_like(Y, 7.0)
    B.bigcn_rms_norm_forward(x, None, EPS, R=r, Y=only)
    assert torch.equal(only, Y)
    B.bigcn_rms_norm_forward(x, None, EPS, R=r, S=only)
    assert torch.equal(only, S)
    alone = torch.full_like(rstd, 7.0)
    B.bigcn_rms_norm_forward(x, None, EPS, R=r, rstd=alone)
    assert torch.equal(alone, rstd)
    q3, e3 = B.checkpoint_buffers(N, K, cuda_device)
    B.bigcn_rms_norm_forward(x, None, EPS, R=r, q=q3, exps=e3)
    assert torch.equal(q3, q) and torch.equal(e3, exps)
    for place in ("R", "X"):
        a, b = x.clone(), r.clone()
        B.bigcn_rms_norm_forward(a, None, EPS, R=b, S=b if place == "R" else a, Y=only, rstd=alone)
        assert torch.equal(b if place == "R" else a, S) and torch.equal(only, Y)
        assert torch.equal(a if place == "R" else b, x if place == "R" else r)
        assert torch.equal(alone, rstd)


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("pad,offset", [(1, 1), (2, 2), (3, 0), (8, 4), (0, 8), (16, 3)])
@pytest.mark.parametrize("K", [64, 98, 203, 1024])
def test_forward_strides_and_offsets(cuda_device, K, pad, offset, dtype):
    """Rows of other strides and alignments; nothing outside the rows is written."""
    N = 35
    x, r = rows(N, K, K + pad, dtype), rows(N, K, K + pad + 1, dtype)
    gamma = params(K, K)[0]
    X, _ = strided(x, pad, offset, cuda_device)
    S, sbuf = strided(r, pad, offset, cuda_device, fill=7.0)        # R, in place
    Y, buf = strided(torch.zeros_like(x), pad, offset, cuda_device, fill=7.0)
    g, _ = strided(torch.from_numpy(gamma)[None], 0, offset, cuda_device)
    rstd = torch.empty(N, device=cuda_device)
    kq, ke = (K + 15) // 16 * 16, ((K + 31) // 32 + 3) // 4 * 4
    qb = torch.full((N + 1, kq + 32), 99, dtype=torch.int8, device=cuda_device)
    eb = torch.full((N + 1, ke + 8), 99, dtype=torch.uint8, device=cuda_device)
    q, exps = qb[:N, :K], eb[:N, :(K + 31) // 32]
    B.bigcn_rms_norm_forward(X, g[0], EPS, R=S, S=S, Y=Y, rstd=rstd, q=q, exps=exps)
    s = summed(x, r)
    assert torch.equal(S.cpu(), s)
    ry, rr, rx = R.rms_forward(f64(s), gamma, EPS)
    ey, er, ex = R.rms_forward_bounds(f64(s), gamma, EPS, dtype)
    within(Y, ry, ey, "Y")
    within(rstd, rr, er, "rstd")
    check_checkpoint(q, exps, rx, ex, K)
    for view, whole in ((Y, buf), (S, sbuf)):
        view.fill_(7.0)
        assert (whole == 7.0).all()
    # Padding up to 16 and 4 bytes is 0, beyond it untouched.
    assert (qb[:N, K:kq] == 0).all() and (qb[:N, kq:] == 99).all() and (qb[N] == 99).all()
    assert (eb[:N, (K + 31) // 32:ke] == 0).all() and (eb[:N, ke:] == 99).all()
    assert (eb[N] == 99).all()


@pytest.mark.parametrize("K", [5, 40, 64, 602, 5000, 9000])
def test_forward_special_rows(cuda_device, K):
    """Tiny and huge rows, at which single squares leave fp32, keep the precision of others; NaN and
    infinity stay in their row; a row of zeros is 0 with an eps and NaN without."""
    x = rows(10, K, 3, "float32").numpy()
    x[0] *= 1e-30
    x[1] *= 1e30
    x[2] *= 2.0 ** -120                 # its square root of squares subnormal but in its inputs normal
    x[3, 1:] *= 1e-20
    x[4, K // 2] = np.nan
    x[5, 0] = np.inf
    x[6, K - 1] = -np.inf
    x[7] = 0.0
    x[8] *= 1e18
    for eps in (0.0, 1e-5, 1e-25):
        Y, _, rstd, q, exps = B.rms_norm_forward(torch.from_numpy(x).to(cuda_device), None, eps)
        fine = [0, 1, 2, 3, 8, 9] + ([7] if eps else [])
        ry, rr, rx = R.rms_forward(x[fine], np.ones(K), eps)
        ey, er, ex = R.rms_forward_bounds(x[fine], np.ones(K), eps, "float32")
        within(Y[fine], ry, ey + 2.0 ** -149, "Y")
        within(rstd[fine], rr, er, "rstd")
        step = np.repeat(2.0 ** (exps[fine].cpu().numpy().astype(float) - 127), 32, axis=1)[:, :K]
        within(N_.values(q[fine].cpu().numpy(), exps[fine].cpu().numpy()), rx, step / 2 + ex + 2.0 ** -149,
               "checkpoint")
        bad = [4, 5, 6] + ([] if eps else [7])
        assert torch.isnan(Y[bad]).all() and (exps[bad] == 255).all()
        if eps:
            assert (Y[7] == 0).all() and (q[7] == 0).all()


def test_half_sum_past_its_range(cuda_device):
    x = torch.full((2, 40), 40000.0, dtype=torch.float16)
    x[1] = 1.0
    r = x.clone()
    Y, S, rstd, q, exps = B.rms_norm_forward(x.to(cuda_device), None, EPS, R=r.to(cuda_device))
    assert torch.isinf(S[0]).all() and torch.isnan(Y[0]).all() and torch.isnan(rstd[0])
    assert (exps[0] == 255).all() and (S[1] == 2.0).all() and not torch.isnan(Y[1]).any()


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("past", [False, True])
@pytest.mark.parametrize("source", ["input", "checkpoint"])
@pytest.mark.parametrize("N,K", SHAPES)
def test_backward(cuda_device, N, K, source, past, dtype):
    s = rows(N, K, 2 * N + K, dtype)
    dy = (0.1 * rows(N, K, 7 * N + K, "float32", level=0.2)).to(DTYPES[dtype])
    ds = (0.1 * rows(N, K, 9 * N + K, "float32", level=0.2)).to(DTYPES[dtype]) if past else None
    gamma = params(K, K + 1)[0]
    _, rr, rx = R.rms_forward(f64(s), gamma, EPS)
    rstd = rr.astype(np.float32)
    t = lambda a: torch.from_numpy(a).to(cuda_device)
    if source == "input":
        shat = f64(s) * rstd[:, None].astype(np.float64)
        kw, ex = dict(S=s.to(cuda_device)), N_.U * np.abs(shat)
    else:
        q, exps = B.checkpoint_pack(t(rx.astype(np.float32)))
        shat, ex = N_.values(q.cpu().numpy(), exps.cpu().numpy()), np.zeros((N, K))
        kw = dict(q=q, exps=exps)
    dX, dg = B.rms_norm_backward(dy.to(cuda_device), t(gamma), t(rstd),
                                 dS=ds.to(cuda_device) if past else None, **kw)
    d64 = f64(ds) if past else 0.0
    rdx, rdg = R.rms_backward(f64(dy), gamma, shat, rstd.astype(np.float64), d64)
    e, eg = R.rms_backward_bounds(f64(dy), gamma, shat, rstd.astype(np.float64), dtype, ex, d64)
    within(dX, rdx, e, "dX")
    within(dg, rdg, eg, "dgamma")


@pytest.mark.parametrize("K", [6, 40, 203])
def test_backward_matches_differences(cuda_device, K):
    """dX and dgamma against central differences of the 64-bit forward: 1e-4 of their scale (the
    differences' own error, h^2, is 1e-8 of it and the fp32 gradient's 1e-6)."""
    N, h = 4, 1e-4
    r = np.random.default_rng(K)
    x, res = rows(N, K, K, "float32"), rows(N, K, K + 1, "float32")
    gamma = params(K, 3)[0]
    dy, ds = (r.standard_normal((N, K)).astype(np.float32) for _ in range(2))
    t = lambda a: torch.from_numpy(a).to(cuda_device)
    _, S, rstd, _, _ = B.rms_norm_forward(x.to(cuda_device), t(gamma), EPS, R=res.to(cuda_device),
                                          checkpoint=False)
    dX, dg = B.rms_norm_backward(t(dy), t(gamma), rstd, S=S, dS=t(ds))

    def loss(s, g):
        return (R.rms_forward(s, g, EPS)[0] * dy).sum() + (s * ds).sum()

    s64, g64 = f64(S), gamma.astype(np.float64)
    for _ in range(6):
        vs, vg = r.standard_normal((N, K)), r.standard_normal(K)
        d = (loss(s64 + h * vs, g64) - loss(s64 - h * vs, g64)) / (2 * h)
        assert abs(d - (f64(dX) * vs).sum()) <= 1e-4 * (np.abs(f64(dX) * vs).sum() + 1e-3)
        d = (loss(s64, g64 + h * vg) - loss(s64, g64 - h * vg)) / (2 * h)
        assert abs(d - (f64(dg) * vg).sum()) <= 1e-4 * np.abs(f64(dg) * vg).sum()


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("pad,offset", [(1, 1), (2, 2), (8, 0), (5, 3)])
@pytest.mark.parametrize("K", [64, 98, 203, 1024])
def test_backward_strides_in_place(cuda_device, K, pad, offset, dtype):
    """dX in the place of dS, in rows of other strides; nothing outside them is written."""
    N = 77
    s, dy, ds = (rows(N, K, K + i, dtype) for i in range(3))
    gamma = params(K, K)[0]
    _, rr, _ = R.rms_forward(f64(s), gamma, EPS)
    t = lambda a: torch.from_numpy(a.astype(np.float32)).to(cuda_device)
    S, _ = strided(s, pad, offset, cuda_device)
    dY, _ = strided(dy, pad, offset, cuda_device)
    dX, buf = strided(ds, pad, offset, cuda_device, fill=7.0)
    ws = torch.empty(B.bigcn_rms_norm_backward_workspace_bytes(N, K), dtype=torch.uint8,
                     device=cuda_device)
    dg, rstd = torch.empty(K, device=cuda_device), t(rr)
    B.bigcn_rms_norm_backward(dY, t(gamma), rstd, ws, S=S, dS=dX, dX=dX, dgamma=dg)
    shat = f64(s) * f64(rstd)[:, None]
    rdx, rdg = R.rms_backward(f64(dy), gamma, shat, f64(rstd), f64(ds))
    e, eg = R.rms_backward_bounds(f64(dy), gamma, shat, f64(rstd), dtype, N_.U * np.abs(shat), f64(ds))
    within(dX, rdx, e, "dX")
    within(dg, rdg, eg, "dgamma")
    dX.fill_(7.0)
    assert (buf == 7.0).all()


@pytest.mark.parametrize("N,K", [(1, 203), (700, 602), (3, 9000), (5000, 64)])
def test_backward_parts(cuda_device, N, K):
    """Each output alone is what it is with the other; repeated calls agree bit for bit; a workspace
    full of NaN changes nothing."""
    dy, ds = (rows(N, K, i, "float32").to(cuda_device) for i in (1, 2))
    gamma = torch.from_numpy(params(K, 2)[0]).to(cuda_device)
    _, _, rstd, q, exps = B.rms_norm_forward(rows(N, K, 3, "float32").to(cuda_device))
    want = B.rms_norm_backward(dy, gamma, rstd, q=q, exps=exps, dS=ds)
    ws = torch.empty(B.bigcn_rms_norm_backward_workspace_bytes(N, K) // 4, device=cuda_device)
    for dx, dg in ((True, True), (True, False), (False, True)):
        ws.fill_(float("nan"))
        X, G = torch.full_like(dy, 7.0), torch.full_like(gamma, 7.0)
        B.bigcn_rms_norm_backward(dy, gamma, rstd, ws if dg else None, q=q, exps=exps,
                                  dS=ds if dx else None, dX=X if dx else None,
                                  dgamma=G if dg else None)
        assert not dx or torch.equal(X, want[0])
        assert not dg or torch.equal(G, want[1])


def test_no_rows(cuda_device):
    e = lambda *s: torch.empty(s, device=cuda_device)
    g = torch.full((5,), 7.0, device=cuda_device)
    B.bigcn_rms_norm_forward(e(0, 5), None, EPS, R=e(0, 5), S=e(0, 5), Y=e(0, 5), rstd=e(0))
    B.bigcn_rms_norm_backward(e(0, 5), None, e(0), torch.empty(256, dtype=torch.uint8, device=cuda_device),
                              S=e(0, 5), dX=e(0, 5), dgamma=g)
    assert (g == 0).all()


def test_other_stream_and_capture(cuda_device):
    """On a stream of its own, and captured and replayed on new inputs in the same buffers."""
    N, K = 300, 203
    x, r, dy = (rows(N, K, i, "bfloat16").to(cuda_device) for i in range(3))
    gamma = torch.from_numpy(params(K, 2)[0]).to(cuda_device)
    Y, S, dX = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x)
    rstd, dg = torch.empty(N, device=cuda_device), torch.empty(K, device=cuda_device)
    q, exps = B.checkpoint_buffers(N, K, cuda_device)
    ws = torch.empty(B.bigcn_rms_norm_backward_workspace_bytes(N, K), dtype=torch.uint8, device=cuda_device)

    def step():
        B.bigcn_rms_norm_forward(x, gamma, EPS, R=r, S=S, Y=Y, rstd=rstd, q=q, exps=exps)
        B.bigcn_rms_norm_backward(dy, gamma, rstd, ws, q=q, exps=exps, dS=r, dX=dX, dgamma=dg)

    outs = (Y, S, dX, rstd, dg)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
        first = [t.clone() for t in outs]
    torch.cuda.current_stream().wait_stream(s)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    x.mul_(-0.5)
    g.replay()
    torch.cuda.synchronize()
    second = [t.clone() for t in outs]
    step()
    assert all(torch.equal(a, b) for a, b in zip(second, outs))
    assert not any(torch.equal(a, b) for a, b in zip(first, second))
    x.mul_(-2.0)
    step()
    assert all(torch.equal(a, b) for a, b in zip(first, outs))
