"""The mean of a row in layer norm's forward. A row's level enters xhat divided by its spread, so
an ulp of the mean of a constant row at 1000 is 0.02 of xhat (eps = 1e-5): the mean has to be the
nearest fp32 number, not a few ulps beside it."""
import numpy as np
import pytest
import torch

import norm_reference as R
from paper_2010_07565_gb300 import binding as B
from test_gpu_norm import DTYPES, EPS, f64, params, rng, within

pytestmark = pytest.mark.gpu

LEVELS = [100.0, 256.0, 1000.0, -1000.0, 0.1, -3.7, 1e-20, 60000.0, 0.0]


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("checkpoint", [False, True])
@pytest.mark.parametrize("N,K", [(9, 1), (9, 3), (9, 41), (9, 47), (9, 500), (9, 1000), (9, 602),
                                 (9, 1433), (9, 5003), (9, 8191), (9, 9001), (9, 20011),
                                 (9000, 41), (9000, 47), (9000, 500), (9000, 602), (9000, 1000)])
def test_constant_rows_are_beta(cuda_device, N, K, checkpoint, dtype):
    """The mean of a constant row is its value, so that xhat is 0 and Y is beta, rounded to the
    type, bit for bit; all groups of the checkpoint are zeros."""
    level = torch.tensor(LEVELS * (N // len(LEVELS))).to(DTYPES[dtype])
    X = level[:, None].expand(N, K).contiguous().to(cuda_device)
    gamma, beta = (torch.from_numpy(p).to(cuda_device) for p in params(K, K))
    Y, mean, rstd, q, exps = B.layer_norm_forward(X, gamma, beta, EPS, checkpoint=checkpoint)
    assert torch.equal(mean.cpu(), level.float())
    assert torch.equal(Y, beta.to(DTYPES[dtype]).expand(N, K))
    # The sum with eps is exact (the variance is 0); a square root, a division, half an ulp each.
    assert np.abs(f64(rstd) * np.sqrt(np.float64(np.float32(EPS))) - 1).max() <= 4 * R.U
    if checkpoint:
        assert (q == 0).all() and (exps == 1).all()


@pytest.mark.parametrize("K", [1, 41, 47, 500, 1433, 9001])
def test_constant_rows_without_eps_are_nan(cuda_device, K):
    """eps = 0: no spread to divide by."""
    X = torch.tensor(LEVELS)[:, None].expand(len(LEVELS), K).contiguous().to(cuda_device)
    Y, mean, rstd, q, exps = B.layer_norm_forward(X, None, None, 0.0)
    assert torch.isnan(Y).all() and torch.isinf(rstd).all() and (exps == 255).all()
    assert torch.equal(mean.cpu(), torch.tensor(LEVELS))


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("N,K", [(40, 2), (40, 41), (7, 47), (40, 500), (2000, 602), (5, 1433),
                                 (3, 5003), (3, 9001), (3, 20011)])
def test_means_of_rows_far_from_zero(cuda_device, N, K, dtype):
    """Rounded once: half an ulp (u of it), beside the error of the deviations' sum. The first sum
    gives a mean within e0 = (D + 2) u mean|x|. What is added to it is the mean of x - mean0, of
    terms rounded once (u), summed in D additions and multiplied by a rounded 1/K (2 u): within
    (D + 4) u mean|x - mean0|, and |x - mean0| <= |x - mean| + e0."""
    r = rng(K)
    x = r.standard_normal((N, K)) * 10.0 ** r.uniform(-2, 1, (N, 1)) + \
        1000.0 * r.choice([-1.0, 1.0], (N, 1)) * r.uniform(0.5, 3.0, (N, 1))
    x = torch.from_numpy(x.astype(np.float32)).to(DTYPES[dtype])
    Y, mean, rstd, _, _ = B.layer_norm_forward(x.to(cuda_device), None, None, EPS, checkpoint=False)
    x = f64(x)
    ref = x.mean(1)
    D = R.row_depth(K)
    e0 = (D + 2) * R.U * np.abs(x).mean(1)
    spread = np.abs(x - ref[:, None]).mean(1)
    within(mean, ref, R.U * np.abs(ref) + (D + 4) * R.U * (spread + e0), "mean")
