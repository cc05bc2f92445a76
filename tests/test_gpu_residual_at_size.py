"""The residual layer's operators where offsets pass 32 bits: the last rows against the 64-bit reference (a
few rows alone lie over more threads, whose sums have another order), or bit for bit what they are
alone where no sum is taken over a row or its order is the same."""
import numpy as np
import pytest
import torch

import norm_reference as N_
import residual_reference as R
from paper_2010_07565_gb300 import binding as B
from test_gpu_norm import f64, within

pytestmark = pytest.mark.gpu

TAIL = 300


def test_rows_past_32_bits(cuda_device):
    """4.3e9 columns of fp16: norm forward and backward, 4 bits and back."""
    N, K = (1 << 21) + 3, 2050
    assert N * K > 1 << 32
    g = torch.Generator(device=cuda_device).manual_seed(3)
    X = torch.empty((N, K), dtype=torch.float16, device=cuda_device)
    for a in range(0, N, 1 << 18):
        X[a:a + (1 << 18)].normal_(generator=g)
    gamma = torch.rand(K, generator=g, device=cuda_device)
    Y, _, rstd, kept, exps = B.rms_norm_forward(X, gamma, R=X)
    last = X[-TAIL:].clone()
    both = f64((last.float() + last.float()).half())
    gam = f64(gamma)
    ry, rr, rx = R.rms_forward(both, gam, 1e-5)
    ey, er, ex = R.rms_forward_bounds(both, gam, 1e-5, "float16")
    within(Y[-TAIL:], ry, ey, "Y")
    within(rstd[-TAIL:], rr, er, "rstd")
    en = exps[-TAIL:].cpu().numpy()
    shat = N_.values(kept[-TAIL:].cpu().numpy(), en)
    step = np.repeat(2.0 ** (en.astype(float) - 127), 32, axis=1)[:, :K]
    within(shat, rx, step / 2 + ex, "checkpoint")
    dX = torch.empty_like(Y)
    B.bigcn_rms_norm_backward(Y, gamma, rstd, None, q=kept, exps=exps, dS=X, dX=dX)
    dy, ds, r = f64(Y[-TAIL:]), f64(last), f64(rstd[-TAIL:])
    rdx, _ = R.rms_backward(dy, gam, shat, r, ds)
    e, _ = R.rms_backward_bounds(dy, gam, shat, r, "float16", np.zeros_like(shat), ds)
    within(dX[-TAIL:], rdx, e, "dX")
    del dX, Y, kept, exps
    q, s = B.fp4_pack(X)
    ql, sl = B.fp4_pack(last)
    assert torch.equal(q[-TAIL:], ql) and torch.equal(s[-TAIL:], sl)
    assert torch.equal(B.fp4_unpack(q, s, K, torch.bfloat16)[-TAIL:], B.fp4_unpack(ql, sl, K, torch.bfloat16))


def test_product_past_32_bits(cuda_device):
    """4.4e9 entries of Z, by tiles of 128 columns and straight stores and not."""
    N, K = (1 << 23) + 17, 70
    g = torch.Generator(device=cuda_device).manual_seed(4)
    a, ae = B.fp4_pack(torch.randn((N, K), generator=g, device=cuda_device))
    for F in (528, 525):
        assert N * F > 1 << 32
        b, be = B.fp4_pack(torch.randn((F, K), generator=g, device=cuda_device))
        Z = B.fp4_gemm(a, ae, b, be, K, dtype=torch.bfloat16)
        assert torch.equal(Z[-TAIL:], B.fp4_gemm(a[-TAIL:], ae[-TAIL:], b, be, K, dtype=torch.bfloat16))
        assert torch.equal(Z[:TAIL], B.fp4_gemm(a[:TAIL], ae[:TAIL], b, be, K, dtype=torch.bfloat16))
        del Z
    assert B.device_timeouts() == 0


def test_a_tensor_past_32_bits(cuda_device):
    """2^32 + 5 ones: the norm is 2^16 to its rounding, and every element is scaled."""
    t = torch.ones((1 << 32) + 5, dtype=torch.bfloat16, device=cuda_device)
    norm = B.clip_grad_norm([t], 2.0 ** 14)
    assert abs(norm.item() - 2.0 ** 16) <= 2.0 ** 16 * 2.0 ** -20
    assert (t[:1 << 20] == 0.25).all() and (t[-(1 << 20):] == 0.25).all()
    assert t.min().item() == 0.25 and t.max().item() == 0.25


def test_two_graphs_in_turn_share_a_workspace(cuda_device):
    """Two captured steps with one workspace, replayed one after the other: each finds only what it wrote."""
    g = torch.Generator(device=cuda_device).manual_seed(5)
    ws = torch.empty(1 << 22, dtype=torch.uint8, device=cuda_device)
    sets, graphs, wants = [], [], []
    for N, K in ((3000, 100), (500, 203)):
        dY, S = (torch.randn((N, K), generator=g, device=cuda_device) for _ in range(2))
        rstd = torch.rand(N, generator=g, device=cuda_device)
        dX, dg, norm = torch.empty_like(dY), torch.empty(K, device=cuda_device), torch.empty(1, device=cuda_device)

        def step(dY=dY, S=S, rstd=rstd, dX=dX, dg=dg, norm=norm):
            B.bigcn_rms_norm_backward(dY, None, rstd, ws, S=S, dX=dX, dgamma=dg)
            B.bigcn_grad_norm([dX, dg], norm, ws)

        step()
        wants.append([t.clone() for t in (dX, dg, norm)])
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        sets.append((dX, dg, norm))
        graphs.append((graph, step))        # (the inputs live with the step)
    for _ in range(3):
        for out, (graph, _) in zip(sets, graphs):
            for t in out:
                t.fill_(float("nan"))
            graph.replay()
    torch.cuda.synchronize()
    for out, want in zip(sets, wants):
        assert all(torch.equal(a, b) for a, b in zip(out, want))
