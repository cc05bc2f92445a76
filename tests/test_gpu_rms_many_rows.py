"""RMS norm, forward and backward, in the layouts that many rows select (several pieces a thread, rows of a warp
and of fewer threads), at every alignment of rows, against the 64-bit bounds."""
import numpy as np
import pytest
import torch

import norm_reference as N_
import residual_reference as R
from paper_2010_07565_gb300 import binding as B
from test_gpu_norm import DTYPES, EPS, MANY, f64, params, rows, strided, within
from test_gpu_rms_norm import check_checkpoint, summed

pytestmark = pytest.mark.gpu

# Widths of every number of pieces a thread, for 8, 16 and 32 threads a row (N above 9728 rows, at which 8 threads
# a row fill the card; 32 do from 2432 on), and rows of 16 bits by a warp with one piece a lane; rows that start at
# 16, 8, 4 and 2 bytes.
WIDTHS = [("float32", 9800, 30, 2, 0), ("float32", 9800, 64, 0, 0), ("float32", 9800, 93, 0, 1),
          ("float32", 9800, 126, 0, 2), ("float32", 9800, 180, 0, 0), ("float32", 9800, 254, 0, 2),
          ("float32", 2500, 380, 0, 0), ("float32", 2500, 511, 0, 0), ("float32", 2500, 640, 0, 0),
          ("float32", 2500, 700, 0, 0), ("float32", 2500, 766, 0, 0), ("float32", 2500, 767, 0, 3),
          ("float32", 2500, 1021, 0, 0),
          ("bfloat16", 9800, 56, 0, 0), ("float16", 9800, 100, 0, 0), ("bfloat16", 9800, 187, 0, 0),
          ("float16", 9800, 190, 0, 2), ("bfloat16", 2500, 250, 0, 0), ("float16", 9800, 250, 6, 0),
          ("bfloat16", 9800, 260, 0, 4), ("float16", 9800, 383, 0, 0), ("bfloat16", 9800, 510, 0, 0),
          ("float16", 2500, 500, 0, 0), ("bfloat16", 2500, 600, 0, 0), ("float16", 2500, 768, 0, 0),
          ("bfloat16", 2500, 767, 0, 5), ("float16", 2500, 766, 0, 0), ("bfloat16", 2500, 1000, 0, 0),
          ("float16", 2500, 1022, 0, 0)]


@pytest.mark.parametrize("dtype,N,K,pad,offset", MANY + WIDTHS)
def test_forward(cuda_device, dtype, N, K, pad, offset):
    """With the addition (in R's place) and the checkpoint, and without either."""
    x, r = rows(N, K, N + K, dtype), rows(N, K, N + K + 1, dtype)
    gamma = params(K, K)[0]
    s = summed(x, r)
    ry, rr, rx = R.rms_forward(f64(s), gamma, EPS)
    ey, er, ex = R.rms_forward_bounds(f64(s), gamma, EPS, dtype)
    X, _ = strided(x, pad, offset, cuda_device)
    S, sbuf = strided(r, pad, offset, cuda_device, fill=7.0)
    Y, buf = strided(torch.zeros_like(x), pad, offset, cuda_device, fill=7.0)
    rstd, alone = (torch.empty(N, device=cuda_device) for _ in range(2))
    g = torch.from_numpy(gamma).to(cuda_device)
    q, exps = B.checkpoint_buffers(N, K, cuda_device)
    B.bigcn_rms_norm_forward(X, g, EPS, R=S, S=S, Y=Y, rstd=rstd, q=q, exps=exps)
    assert torch.equal(S.cpu(), s)
    within(Y, ry, ey, "Y")
    within(rstd, rr, er, "rstd")
    check_checkpoint(q, exps, rx, ex, K)
    first = Y.clone()
    Y.fill_(5.0)
    B.bigcn_rms_norm_forward(S, g, EPS, Y=Y, rstd=alone)
    assert torch.equal(Y, first) and torch.equal(alone, rstd)
    q2, exps2 = B.checkpoint_buffers(N, K, cuda_device)
    B.bigcn_rms_norm_forward(S, g, EPS, q=q2, exps=exps2)
    assert torch.equal(q, q2) and torch.equal(exps, exps2)
    for view, whole in ((Y, buf), (S, sbuf)):
        view.fill_(7.0)
        assert (whole == 7.0).all()


@pytest.mark.parametrize("source", ["input", "checkpoint"])
@pytest.mark.parametrize("dtype,N,K,pad,offset", MANY + WIDTHS)
def test_backward(cuda_device, dtype, N, K, pad, offset, source):
    """With dS (dX in its place) and without."""
    s = rows(N, K, 2 * N + K, dtype)
    dy, ds = ((0.1 * rows(N, K, n * N + K, "float32", level=0.2)).to(DTYPES[dtype]) for n in (7, 9))
    gamma = params(K, K + 1)[0]
    _, rr, rx = R.rms_forward(f64(s), gamma, EPS)
    t = lambda a: torch.from_numpy(a.astype(np.float32)).to(cuda_device)
    rstd = t(rr)
    if source == "input":
        shat = f64(s) * f64(rstd)[:, None]
        kw, ex = dict(S=strided(s, pad, offset, cuda_device)[0]), N_.U * np.abs(shat)
    else:
        q, exps = B.checkpoint_pack(t(rx))
        shat, ex = N_.values(q.cpu().numpy(), exps.cpu().numpy()), np.zeros((N, K))
        kw = dict(q=q, exps=exps)
    dY, _ = strided(dy, pad, offset, cuda_device)
    ws = torch.empty(B.bigcn_rms_norm_backward_workspace_bytes(N, K), dtype=torch.uint8, device=cuda_device)
    g64, r64 = f64(dy), f64(rstd)
    for past in (False, True):
        dX, buf = strided(ds, pad, offset, cuda_device, fill=7.0)
        dg = torch.empty(K, device=cuda_device)
        B.bigcn_rms_norm_backward(dY, t(gamma), rstd, ws, dS=dX if past else None, dX=dX, dgamma=dg, **kw)
        d64 = f64(ds) if past else 0.0
        rdx, rdg = R.rms_backward(g64, gamma, shat, r64, d64)
        e, eg = R.rms_backward_bounds(g64, gamma, shat, r64, dtype, ex, d64)
        within(dX, rdx, e, "dX")
        within(dg, rdg, eg, "dgamma")
        dX.fill_(7.0)
        assert (buf == 7.0).all()
