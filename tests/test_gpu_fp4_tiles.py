"""The 4-bit product in the tile shapes that many rows select: 256 columns with one accumulator, and B's stages
kept in shared memory, each with several tiles a CTA, partial tiles and every kind of store."""
import pytest
import torch

import residual_reference as R
from paper_2010_07565_gb300 import binding as B
from test_gpu_fp4 import values, wide_rows
from test_gpu_norm import DTYPES, rows, strided, within

pytestmark = pytest.mark.gpu


def tile_shape(N, K, F, sms):
    """(columns of a tile, whether B is kept) as bigcn_fp4_gemm chooses them."""
    mt, groups = -(-N // 128), -(-K // 32)
    nt = 256 if F > 128 and K > 2048 and -(-F // 128) % 2 == 0 else 128 if F > 64 else 64 if F > 32 else 32
    while nt > 32 and mt * -(-F // nt) * 2 <= sms:
        nt //= 2
    return nt, nt in (64, 128) and F <= nt and groups <= 24 and mt > sms


CASES = [(10300, 2050, 500, (256, False)),      # 162 tiles: some CTAs take two
         (20000, 2080, 256, (256, False)),
         (10111, 4100, 200, (256, False)),
         (20011, 768, 128, (128, True)),
         (45001, 602, 100, (128, True)),
         (19999, 70, 65, (128, True)),
         (20011, 800, 128, (128, False)),
         (20011, 768, 64, (64, True)),
         (60001, 602, 41, (64, True)),
         (19999, 33, 40, (64, True)),
         (20011, 800, 50, (64, False)),
         (20011, 602, 7, (32, False))]


@pytest.mark.parametrize("N,K,F,shape", CASES)
def test_tiles(cuda_device, N, K, F, shape):
    sms = torch.cuda.get_device_properties(cuda_device).multi_processor_count
    assert tile_shape(N, K, F, sms) == shape
    b = B.fp4_pack(rows(F, K, F + K, "float32").to(cuda_device))
    bias = rows(1, F, 9, "float32")[0]
    vb = values(*b, K)
    for wide in (True, False):              # (rows of one level are within fp16's range)
        x = wide_rows(N, K, N + K, "float32") if wide else rows(N, K, 5, "float32")
        a = B.fp4_pack(x.to(cuda_device))
        va = values(*a, K)
        for with_bias in (False, True):
            c = bias.double().numpy() if with_bias else 0.0
            ref = R.fp4_gemm(va, vb, c)
            for dtype in ("float32", "bfloat16") if wide else ("float16",):
                bound = R.fp4_gemm_bounds(va, vb, c, dtype)
                for pad, offset in ((0, 0), (-F % 16, 0), (1, 3)):
                    Z, buf = strided(torch.zeros(N, F, dtype=DTYPES[dtype]), pad, offset, cuda_device, fill=7.0)
                    B.bigcn_fp4_gemm(*a, *b, K, Z, bias.to(cuda_device) if with_bias else None)
                    within(Z, ref, bound, f"Z {dtype} {pad} {with_bias}")
                    Z.fill_(7.0)
                    assert (buf == 7.0).all()
    assert B.device_timeouts() == 0


@pytest.mark.parametrize("N,K,F", [(20000, 2080, 256), (20011, 602, 128), (20011, 602, 64)])
def test_rows_are_the_same_bits_in_other_tiles(cuda_device, N, K, F):
    """A row's products alone (tiles of 32 columns) and in the shapes above; repeated calls too."""
    a = B.fp4_pack(wide_rows(N, K, 3, "float32").to(cuda_device))
    b = B.fp4_pack(rows(F, K, 4, "float32").to(cuda_device))
    Z = B.fp4_gemm(*a, *b, K)
    assert torch.equal(Z, B.fp4_gemm(*a, *b, K))
    for i in (0, 129, 19456, N - 1):
        assert torch.equal(B.fp4_gemm(a[0][i:i + 1], a[1][i:i + 1], *b, K), Z[i:i + 1])
    assert B.device_timeouts() == 0


@pytest.mark.parametrize("N,K,F", [(20000, 2080, 256), (20011, 602, 128), (20011, 602, 64)])
def test_nan_groups_in_these_tiles(cuda_device, N, K, F):
    """NaN groups reach the sums that they are part of and no others, where a CTA goes on to more tiles."""
    q, e = B.fp4_pack(rows(N, K, 3, "float32").to(cuda_device))
    b = B.fp4_pack(rows(F, K, 4, "float32").to(cuda_device))
    Z = B.fp4_gemm(q, e, *b, K)
    at = torch.tensor([0, 200, 19456, N - 1], device=cuda_device)
    e[at, -1] = 255
    q[at, (e.shape[1] - 1) * 16:] = 0
    bad = torch.zeros(N, dtype=torch.bool, device=cuda_device)
    bad[at] = True
    got = B.fp4_gemm(q, e, *b, K)
    assert torch.isnan(got[bad]).all() and torch.equal(got[~bad], Z[~bad])
    assert B.device_timeouts() == 0
