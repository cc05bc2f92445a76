"""RMS norm of rows whose root mean square is so small that its reciprocal passes fp32's range."""
import numpy as np
import pytest
import torch

import norm_reference as N_
import residual_reference as R
from paper_2010_07565_gb300 import binding as B
from test_gpu_norm import DTYPES, f64, within

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("eps", [0.0, 1e-38, 1e-30])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("K", [5, 40, 64, 300, 602, 1000, 5000, 9000, 20000])
def test_rows_below_the_range_of_rstd(cuda_device, K, dtype, eps):
    """Without an eps a row of subnormals is normalised like any other, though its rstd is infinite in fp32;
    the stream keeps it as it is."""
    least = 2.0 ** (-149 if dtype == "float32" else -133)
    r = np.random.default_rng(K)
    x = r.standard_normal((8, K)).astype(np.float32)
    x[0] = 2.0 ** -131 * r.choice([-1.0, 1.0], K)
    x[1] = least * r.integers(1, 8, K) * r.choice([-1.0, 1.0], K)
    x[2] = 0.0
    x[2, K // 2] = -least
    x[4] = 2.0 ** -129
    x[5] = 2.0 ** -127
    x[6] *= 2.0 ** -100
    x[7, 1:] *= 2.0 ** -120
    x = torch.from_numpy(x).to(DTYPES[dtype])
    zeros, S, Y = torch.zeros_like(x).to(cuda_device), *(torch.empty_like(x).to(cuda_device) for _ in range(2))
    rstd = torch.empty(8, device=cuda_device)
    q, exps = B.checkpoint_buffers(8, K, cuda_device)
    B.bigcn_rms_norm_forward(x.to(cuda_device), None, eps, R=zeros, S=S, Y=Y, rstd=rstd, q=q, exps=exps)
    assert torch.equal(S.cpu(), x)
    e32 = float(np.float32(eps))
    ry, rr, rx = R.rms_forward(f64(x), np.ones(K), e32)
    ey, er, ex = R.rms_forward_bounds(f64(x), np.ones(K), e32, dtype)
    within(Y, ry, ey + 2.0 ** -149, "Y")
    past = rr > np.finfo(np.float32).max
    assert past.sum() == (4 if eps == 0 else 0)
    got = f64(rstd)
    assert np.isposinf(got[past]).all()
    within(got[~past], rr[~past], er[~past], "rstd")
    en = exps.cpu().numpy()
    step = np.repeat(2.0 ** (en.astype(float) - 127), 32, axis=1)[:, :K]
    within(N_.values(q.cpu().numpy(), en), rx, step / 2 + ex + 2.0 ** -149, "checkpoint")
