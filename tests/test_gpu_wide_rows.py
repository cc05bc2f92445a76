"""The norms of rows so wide that one running fp32 sum a thread would not hold their sums."""
import numpy as np
import pytest
import torch

import norm_reference as N_
from norm_reference import U
from paper_2010_07565_gb300 import binding as B
from test_gpu_norm import DTYPES

pytestmark = pytest.mark.gpu

# Additions that a term of a wide row's sum passes in fp32: a run of 256, the block's 5 and 8 behind it, and
# two roundings of what is held in 64 bits.
DEPTH = 256 + 15
WIDE = (1 << 24) + 77


@pytest.mark.parametrize("level", [1.1, 1.1 * 2.0 ** -70, 1.1 * 2.0 ** 60])
def test_rms_norm_of_a_wide_row(cuda_device, level):
    """Equal values: the roundings of a running sum are all of one sign."""
    v = float(np.float32(level))
    x = torch.full((1, WIDE), v, device=cuda_device)
    Y, _, rstd, _, _ = B.rms_norm_forward(x, None, 0.0, checkpoint=False)
    error = (0.5 * (DEPTH + 4) + 3) * U
    assert abs(rstd.item() * v - 1) <= error
    assert (Y - 1).abs().max().item() <= error + 2 * U


def test_rms_norm_backward_of_a_wide_row(cuda_device):
    """dy and shat of one value each: dx is what their mean leaves of g."""
    s, dy = float(np.float32(1.1)), float(np.float32(0.3))
    S, dY = (torch.full((1, WIDE), v, device=cuda_device) for v in (s, dy))
    rstd = torch.tensor([0.9], device=cuda_device)
    dX, _ = B.rms_norm_backward(dY, None, rstd, S=S)
    r = float(np.float32(0.9))
    shat = s * r
    want = r * (dy - shat * dy * shat)
    error = r * dy * (shat * shat * (DEPTH + 6) + 6) * U
    assert (dX.double() - want).abs().max().item() <= error


def two_values(dtype, K, device):
    """A row of a, b, a, b, ...; its mean and variance, in 64 bits."""
    pair = torch.tensor([1.6, 0.6]).to(dtype)
    a, b = pair.double().tolist()
    x = pair.to(device).repeat((K + 1) // 2)[:K][None].contiguous()
    share = ((K + 1) // 2) / K
    mean = b + share * (a - b)
    return x, a, b, mean, share * (1 - share) * (a - b) ** 2


# Likewise for layer norm, whose mean and variance are those of d = x - m0 (rounded, as K and 1 / K are).
@pytest.mark.parametrize("dtype,K", [("float32", WIDE), ("bfloat16", (1 << 29) + (1 << 20))])
def test_layer_norm_of_a_wide_row(cuda_device, dtype, K):
    x, a, b, mean, variance = two_values(DTYPES[dtype], K, cuda_device)
    Y, m, rstd, _, _ = B.layer_norm_forward(x, None, None, 0.0, checkpoint=False)
    off_mean = 2 * U * mean + (DEPTH + 6) * U * (a - b) / 2
    assert abs(m.item() - mean) <= off_mean
    error = (0.5 * (DEPTH + 8) + 6) * U
    assert abs(rstd.item() * np.sqrt(variance) - 1) <= error
    for first, v in ((0, a), (1, b)):
        want = (v - mean) / np.sqrt(variance)
        off = abs(want) * (error + N_.OUT_ROUND[dtype][0]) + off_mean / np.sqrt(variance)
        for at in (0, K // 2 // 2 * 2, K - 4096 - K % 2):
            assert (Y[0, at + first:at + 4096:2].double() - want).abs().max().item() <= 1.01 * off


def test_layer_norm_backward_of_a_wide_row(cuda_device):
    x, a, b, mean, variance = two_values(torch.float32, WIDE, cuda_device)
    dy = float(np.float32(0.3))
    dY = torch.full((1, WIDE), dy, device=cuda_device)
    m, r = (float(np.float32(v)) for v in (mean, 1 / np.sqrt(variance)))
    dX, _, _ = B.layer_norm_backward(dY, None, torch.tensor([r], device=cuda_device), X=x,
                                     mean=torch.tensor([m], device=cuda_device))
    share = ((WIDE + 1) // 2) / WIDE
    ha, hb = (a - m) * r, (b - m) * r
    c1 = dy * (share * ha + (1 - share) * hb)
    size = dy * (share * abs(ha) + (1 - share) * abs(hb))
    for first, h in ((0, ha), (1, hb)):
        want = r * (dy - dy - h * c1)
        error = r * ((DEPTH + 6) * U * (dy + abs(h) * size) + 6 * U * (dy + abs(h) * abs(c1)))
        assert (dX[0, first::2].double() - want).abs().max().item() <= error
