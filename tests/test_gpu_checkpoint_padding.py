"""The bytes behind a checkpoint's row, up to K rounded up to 16, are 0 whatever the row holds, a NaN
and an infinity among it; a group that holds one has q = 0 throughout."""
import pytest
import torch

from paper_2010_07565_gb300 import binding as B
from test_gpu_norm import DTYPES, EPS, rows

pytestmark = pytest.mark.gpu

# Rows in registers by 8 threads up to 512, and rows too long for that; 1 to 15 bytes of padding.
SHAPES = [(40, 1), (40, 33), (5000, 41), (40, 203), (40, 602), (9, 1433), (6, 5003), (6, 9001),
          (6, 20011)]


def special(N, K, dtype):
    x = rows(N, K, N + K, dtype)
    x[1, K - 1], x[2, K - 1], x[3, 0] = float("nan"), float("inf"), -float("inf")
    x[4, K // 2] = float("nan")
    return x


def buffers(N, K, device):
    kq = (K + 15) // 16 * 16
    qb = torch.full((N, kq + 16), 99, dtype=torch.int8, device=device)
    groups = (K + 31) // 32
    eb = torch.full((N, (groups + 3) // 4 * 4 + 4), 99, dtype=torch.uint8, device=device)
    return qb, eb, qb[:, :K], eb[:, :groups]


def check(qb, eb, K, nan_groups):
    kq, groups = (K + 15) // 16 * 16, (K + 31) // 32
    ke = (groups + 3) // 4 * 4
    assert (qb[:, K:kq] == 0).all() and (qb[:, kq:] == 99).all()
    assert (eb[:, groups:ke] == 0).all() and (eb[:, ke:] == 99).all()
    assert torch.equal(eb[:, :groups] == 255, nan_groups)
    wide = nan_groups.repeat_interleave(32, 1)[:, :K]
    assert (qb[:, :K][wide] == 0).all()


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("N,K", SHAPES)
def test_padding_of_packed_rows(cuda_device, N, K, dtype):
    X = special(N, K, dtype).to(cuda_device)
    qb, eb, q, exps = buffers(N, K, cuda_device)
    B.bigcn_checkpoint_pack(X, q, exps)
    bad = torch.nn.functional.pad(~torch.isfinite(X), (0, -K % 32)).view(N, -1, 32).any(2)
    check(qb, eb, K, bad)


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("N,K", SHAPES)
def test_padding_of_normalised_rows(cuda_device, N, K, dtype):
    X = special(N, K, dtype).to(cuda_device)
    qb, eb, q, exps = buffers(N, K, cuda_device)
    B.bigcn_layer_norm_forward(X, None, None, EPS, torch.empty_like(X), q=q, exps=exps)
    bad = (~torch.isfinite(X)).any(1, keepdim=True).expand(N, (K + 31) // 32)
    check(qb, eb, K, bad)
