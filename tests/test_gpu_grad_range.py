"""fp32 gradients of any size in the weight gradient: three bf16 parts hold all 24 bits above 2^-110,
and below to half of bf16's least subnormal, 2^-133; fp16 and bf16 gradients down to their own least."""
import numpy as np
import pytest
import torch

from paper_2010_07565_gb300 import binding as B
from test_gpu_norm import f64, rng, within

pytestmark = pytest.mark.gpu


def one_row(dz, power, device):
    """dW of one row of features 64 * 2^power: 64 * 2^power * dz, a single product for each entry."""
    F = dz.shape[1]
    q, exps = B.checkpoint_buffers(1, 32, device)
    q.fill_(64), exps.fill_(127 + power)
    dW, db = B.checkpoint_weight_grad(q, exps, dz.to(device))
    return f64(dW) * 2.0 ** -(power + 6), f64(db)


@pytest.mark.parametrize("F", [64, 41])
def test_fp32_gradients_of_any_size(cuda_device, F):
    """One row: the three products of an entry's parts are added without rounding as long as their 24
    bits fit the accumulator, so the parts' own error is all there is."""
    for e in list(range(-109, 30, 9)) + list(range(-149, -109)):
        dz = torch.from_numpy((rng(e + 200).uniform(1, 2, (1, F)) * 2.0 ** e).astype(np.float32))
        got, db = one_row(dz, 100 if e < 0 else 0, cuda_device)
        exact = 2.0 ** -134 if e < -110 else 0.0
        within(got, np.broadcast_to(f64(dz), (32, F)), np.full((32, F), exact), f"2^{e}")
        assert np.array_equal(db, f64(dz)[0])


@pytest.mark.parametrize("dtype,least", [(torch.bfloat16, -133), (torch.float16, -24)])
def test_16_bit_gradients_down_to_the_least(cuda_device, dtype, least):
    dz = torch.tensor([[2.0 ** least * m for m in range(1, 42)]], dtype=dtype)
    got, db = one_row(dz, 100 if least < -100 else 0, cuda_device)
    assert np.array_equal(got, np.broadcast_to(f64(dz), (32, 41))) and np.array_equal(db, f64(dz)[0])
