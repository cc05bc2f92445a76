"""Sums over rows take every row once: whole-number gradients and features, whose products and
sums fp32 (and the tensor cores) hold exactly, so that a lost or doubled row shows in any column
that it is not zero in. The bounds on real data cannot show one row of tens of thousands."""
import numpy as np
import pytest
import torch

from paper_2010_07565_gb300 import binding as B
from test_gpu_norm import DTYPES, MANY, f64, rng, strided

MOST = 3                  # magnitudes of both factors


def whole(N, cols, seed):
    """Whole numbers in [-3, 3], no row of them all zeros."""
    x = rng(seed).integers(-MOST, MOST + 1, (N, cols))
    x[np.arange(N), np.arange(N) % cols] |= 1
    return x


def exact(N):
    """Partial sums of N products stay below 2^24, in whatever order."""
    return N * MOST * MOST < 1 << 24


def kept(v, device):
    """Whole numbers as a checkpoint of step 1."""
    q, exps = B.checkpoint_buffers(*v.shape, device)
    q.copy_(torch.from_numpy(v.astype(np.int8)))
    exps.fill_(127)
    return q, exps


def test_a_row_lost_or_doubled_shows():
    """On the reference: leaving any one row out, or taking it twice, moves the sums."""
    N, K = 700, 40
    dy, v = whole(N, K, 1), whole(N, K, 2)
    assert exact(40007) and (np.abs(dy) <= MOST).all() and (dy != 0).any(1).all()
    db = dy.sum(0)
    for r in range(N):
        assert not np.array_equal(db - dy[r], db) and not np.array_equal(db + dy[r], db)
    moved = sum(not np.array_equal((dy * v).sum(0) - dy[r] * v[r], (dy * v).sum(0)) for r in range(N))
    assert moved == N


@pytest.mark.gpu
@pytest.mark.parametrize("source", ["input", "checkpoint"])
@pytest.mark.parametrize("dtype,N,K,pad,offset", MANY + [
    ("float32", 1, 64, 0, 0), ("float32", 303, 602, 0, 0), ("float16", 2433, 500, 0, 0),
    ("bfloat16", 4865, 256, 0, 0), ("float32", 305, 9001, 0, 0), ("bfloat16", 257, 20011, 0, 0),
    ("float32", 40007, 7, 0, 0), ("float16", 40001, 33, 1, 1), ("float32", 2431, 700, 0, 0)])
def test_parameter_gradients(cuda_device, dtype, N, K, pad, offset, source):
    assert exact(N)
    dy, v = whole(N, K, N + K), whole(N, K, N + 3 * K + 1)
    dY, _ = strided(torch.from_numpy(dy).to(DTYPES[dtype]), pad, offset, cuda_device)
    rstd = torch.ones(N, device=cuda_device)
    if source == "input":       # xhat = (x - mean) 1, in whole numbers
        mean = torch.from_numpy((np.arange(N) % 7 - 3).astype(np.float32))
        X, _ = strided((torch.from_numpy(v) + mean[:, None]).to(DTYPES[dtype]), pad, offset, cuda_device)
        kw = dict(X=X, mean=mean.to(cuda_device))
    else:
        q, exps = kept(v, cuda_device)
        kw = dict(q=q, exps=exps)
    _, dg, db = B.layer_norm_backward(dY, None, rstd, **kw)
    assert np.array_equal(f64(dg), (dy * v).sum(0)) and np.array_equal(f64(db), dy.sum(0))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("N,K,F", [(1, 40, 3), (63, 128, 64), (65, 203, 41), (2708, 1433, 7),
                                   (2708, 1433, 64), (9729, 300, 128), (20011, 96, 41),
                                   (20011, 520, 256), (40001, 130, 3), (40007, 128, 100),
                                   (33333, 260, 192)])
def test_weight_gradient(cuda_device, N, K, F, dtype):
    assert exact(N)
    v, dz = whole(N, K, N + F), whole(N, F, N + 3 * F + 1)
    q, exps = kept(v, cuda_device)
    dW, db = B.checkpoint_weight_grad(q, exps, torch.from_numpy(dz).to(DTYPES[dtype]).to(cuda_device))
    ref = v.astype(np.float64).T @ dz.astype(np.float64)
    assert np.array_equal(f64(dW), ref) and np.array_equal(f64(db), dz.sum(0))
    assert B.device_timeouts() == 0
