"""The weight gradient from an 8-bit checkpoint on the GPU against the 64-bit reference."""
import numpy as np
import pytest
import torch

import norm_reference as R
from paper_2010_07565_gb300 import binding as B
from test_gpu_norm import DTYPES, f64, params, rng, strided, within

pytestmark = pytest.mark.gpu


def case(N, K, F, dtype, seed, device):
    r = rng(seed)
    v = r.standard_normal((N, K)).astype(np.float32)
    dz = (0.1 * r.standard_normal((N, F)) * np.exp(r.standard_normal((N, 1)))).astype(np.float32)
    q, exps = B.checkpoint_pack(torch.from_numpy(v).to(device))
    dz = torch.from_numpy(dz).to(DTYPES[dtype])
    return q, exps, R.values(q.cpu().numpy(), exps.cpu().numpy()), dz


def check(dW, db, v, gamma, beta, dz, what=""):
    rw, rb = R.weight_grad(v, gamma, beta, dz)
    ew, eb = R.weight_grad_bounds(v, gamma, beta, dz)
    within(dW, rw, ew, what + " dW")
    within(db, rb, eb, what + " db")
    if dW.numel() >= 64 and dz.shape[0] >= 256:
        # In the 2-norm: 40 truncations of half an ulp on average on the way of a partial sum
        # (2/3 of 40 half-ulps of 2^-23 to 2^-24), and rounded sums of some hundred parts.
        assert np.linalg.norm(f64(dW) - rw) <= 4e-6 * np.linalg.norm(rw), what


SHAPES = [(1, 1, 1), (2, 3, 5), (31, 32, 7), (33, 33, 64), (64, 128, 41), (65, 130, 65),
          (100, 203, 19), (257, 64, 128), (300, 602, 41), (511, 129, 130), (1000, 500, 3),
          (2708, 1433, 64), (1025, 256, 256), (777, 640, 250), (4000, 300, 129), (640, 70, 300),
          (1500, 1000, 96), (129, 4096, 256), (20000, 128, 8), (30011, 96, 72), (96, 520, 512)]


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("N,K,F", SHAPES)
def test_weight_grad(cuda_device, N, K, F, dtype):
    q, exps, v, dz = case(N, K, F, dtype, N + K + F, cuda_device)
    gamma, beta = params(K, F)
    t = lambda a: torch.from_numpy(a).to(cuda_device)
    dW, db = B.checkpoint_weight_grad(q, exps, dz.to(cuda_device), t(gamma), t(beta))
    check(dW, db, v, gamma, beta, f64(dz), f"{N}x{K}x{F}")
    again = B.checkpoint_weight_grad(q, exps, dz.to(cuda_device), t(gamma), t(beta))
    assert torch.equal(dW, again[0]) and torch.equal(db, again[1])
    assert B.device_timeouts() == 0


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("pad,offset", [(0, 1), (1, 0), (3, 2), (4, 4), (8, 8), (16, 3)])
@pytest.mark.parametrize("F", [8, 41, 64, 100, 256])
def test_weight_grad_strides(cuda_device, F, pad, offset, dtype):
    """Gradient rows of any stride and offset; dW in rows of its own stride, its padding kept;
    what lies between the rows is NaN and never read into a result."""
    N, K = 333, 203
    q, exps, v, dz = case(N, K, F, dtype, F + pad, cuda_device)
    dZ, _ = strided(dz, pad, offset, cuda_device)
    dWv, buf = strided(torch.zeros(K, F), pad, offset, cuda_device, fill=7.0)
    db = torch.empty(F, device=cuda_device)
    ws = torch.empty(B.bigcn_checkpoint_weight_grad_workspace_bytes(N, K, F), dtype=torch.uint8,
                     device=cuda_device)
    B.bigcn_checkpoint_weight_grad(q, exps, dZ, ws, dWv, db=db)
    check(dWv, db, v, np.ones(K), np.zeros(K), f64(dz))
    dWv.fill_(7.0)
    assert (buf == 7.0).all()


def test_weight_grad_padding_of_the_checkpoint_is_ignored(cuda_device):
    N, K, F = 90, 203, 24
    q, exps, v, dz = case(N, K, F, "float32", 1, cuda_device)
    want = B.checkpoint_weight_grad(q, exps, dz.to(cuda_device))
    qb = torch.full((N, 288), 77, dtype=torch.int8, device=cuda_device)
    eb = torch.full((N, 12), 255, dtype=torch.uint8, device=cuda_device)
    qb[:, :K], eb[:, :7] = q, exps
    got = B.checkpoint_weight_grad(qb[:, :K], eb[:, :7], dz.to(cuda_device))
    assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1])
    y1 = B.checkpoint_unpack(q, exps)
    assert torch.equal(y1, B.checkpoint_unpack(qb[:, :K], eb[:, :7]))


def test_weight_grad_scales_and_special_values(cuda_device):
    """Groups of very unlike scales; NaN groups and NaN gradients reach what sums over them and
    nothing else; a gradient of zeros."""
    N, K, F = 700, 256, 40
    r = rng(3)
    x = (r.standard_normal((N, K)) * 10.0 ** r.integers(-18, 18, (N, 1))).astype(np.float32)
    x[:, 64:96] *= np.float32(1e-12)
    q, exps = B.checkpoint_pack(torch.from_numpy(x).to(cuda_device))
    v = R.values(q.cpu().numpy(), exps.cpu().numpy())
    dz = r.standard_normal((N, F)).astype(np.float32)
    dW, db = B.checkpoint_weight_grad(q, exps, torch.from_numpy(dz).to(cuda_device))
    rw, _ = R.weight_grad(v, np.ones(K), np.zeros(K), dz.astype(np.float64))
    ew, _ = R.weight_grad_bounds(v, np.ones(K), np.zeros(K), dz.astype(np.float64))
    within(dW, rw, ew, "dW")
    zero = B.checkpoint_weight_grad(q, exps, torch.zeros((N, F), device=cuda_device))
    assert (zero[0] == 0).all() and (zero[1] == 0).all()
    x = r.standard_normal((N, K)).astype(np.float32)
    x[5, 33] = np.nan
    q, exps = B.checkpoint_pack(torch.from_numpy(x).to(cuda_device))
    dW, db = B.checkpoint_weight_grad(q, exps, torch.from_numpy(dz).to(cuda_device))
    assert torch.isnan(dW[32:64]).all() and torch.isfinite(db).all()
    assert torch.isfinite(dW[:32]).all() and torch.isfinite(dW[64:]).all()
    dz[9, 7] = np.nan
    dW, db = B.checkpoint_weight_grad(q[10:], exps[10:], torch.from_numpy(dz).to(cuda_device)[10:])
    assert torch.isfinite(dW).all() and torch.isfinite(db).all()
    dW, db = B.checkpoint_weight_grad(q[6:], exps[6:], torch.from_numpy(dz).to(cuda_device)[6:])
    others = [j for j in range(F) if j != 7]
    assert torch.isnan(dW[:, 7]).all() and torch.isfinite(dW[:, others]).all()
    assert torch.isnan(db[7]) and torch.isfinite(db[others]).all()


def test_weight_grad_no_rows_and_other_stream(cuda_device):
    K, F = 40, 9
    q, exps = B.checkpoint_buffers(0, K, cuda_device)
    dW, db = torch.ones((K, F), device=cuda_device), torch.ones(F, device=cuda_device)
    B.bigcn_checkpoint_weight_grad(q, exps, torch.empty((0, F), device=cuda_device), None, dW, db=db)
    assert (dW == 0).all() and (db == 0).all()
    q, exps, v, dz = case(3000, 300, 100, "float32", 8, cuda_device)
    dZ = dz.to(cuda_device)
    want = B.checkpoint_weight_grad(q, exps, dZ)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    ws = torch.empty(B.bigcn_checkpoint_weight_grad_workspace_bytes(3000, 300, 100),
                     dtype=torch.uint8, device=cuda_device)
    dW, db = torch.empty((300, 100), device=cuda_device), torch.empty(100, device=cuda_device)
    B.bigcn_checkpoint_weight_grad(q, exps, dZ, ws, dW, db=db, stream=s)
    s.synchronize()
    assert torch.equal(dW, want[0]) and torch.equal(db, want[1])


def test_weight_grad_matches_differences(cuda_device):
    """Directional central differences of the 64-bit product's loss: linear in W and b, so the
    difference is exact but for 64-bit rounding, and the fp32 gradient within 1e-5."""
    N, K, F = 400, 70, 12
    q, exps, v, dz = case(N, K, F, "float32", 4, cuda_device)
    gamma, beta = params(K, 6)
    t = lambda a: torch.from_numpy(a).to(cuda_device)
    dW, db = B.checkpoint_weight_grad(q, exps, dz.to(cuda_device), t(gamma), t(beta))
    y, g = gamma * v + beta, f64(dz)
    r = rng(9)
    W, b = r.standard_normal((K, F)), r.standard_normal(F)
    loss = lambda W, b: ((y @ W + b) * g).sum()
    for _ in range(4):
        dw, dbv = r.standard_normal((K, F)), r.standard_normal(F)
        d = (loss(W + 1e-3 * dw, b) - loss(W - 1e-3 * dw, b)) / 2e-3
        assert abs(d - (f64(dW) * dw).sum()) <= 1e-5 * np.abs(f64(dW) * dw).sum()
        d = (loss(W, b + 1e-3 * dbv) - loss(W, b - 1e-3 * dbv)) / 2e-3
        assert abs(d - (f64(db) * dbv).sum()) <= 1e-5 * np.abs(f64(db) * dbv).sum()


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("N,K,F", [(700, 260, 192), (333, 640, 192), (1000, 520, 320), (65, 40, 448),
                                   (1, 600, 192), (130, 1100, 704)])
def test_weight_grad_boxes_past_the_last_column(cuda_device, N, K, F, dtype):
    """F a multiple of 64, the width of a copied part of dZ's rows, but not of the column tile: the
    last box reaches past F. Rows with a stride above F, whose padding is NaN, and without one."""
    q, exps, v, dz = case(N, K, F, dtype, N + F, cuda_device)
    for pad in (0, 16):
        dZ, _ = strided(dz, pad, 0, cuda_device)
        dW, db = B.checkpoint_weight_grad(q, exps, dZ)
        check(dW, db, v, np.ones(K), np.zeros(K), f64(dz), f"{N}x{K}x{F}+{pad}")
    assert B.device_timeouts() == 0
