"""Rows in microscaled 4 bits and their product on the GPU: packing and reading back exact, the product
within the bound that residual_reference derives."""
import numpy as np
import pytest
import torch

import residual_reference as R
from paper_2010_07565_gb300 import binding as B
from test_gpu_norm import DTYPES, f64, rows, strided, within

pytestmark = pytest.mark.gpu

SHAPES = [(1, 1), (3, 2), (1, 33), (2, 7), (5, 31), (33, 32), (300, 65), (64, 203), (501, 256), (37, 500),
          (333, 602), (19, 1000), (10, 1026), (5, 1433), (4, 2049), (3, 4096), (6, 5003), (2, 8200),
          (1, 70001)]


def same(got, ref):
    """Equal, NaN for NaN; a zero's sign apart."""
    got = got.cpu().double().numpy() if isinstance(got, torch.Tensor) else got
    assert got.shape == ref.shape
    bad = ~((got == ref) | (np.isnan(got) & np.isnan(ref)))
    assert not bad.any(), (np.argwhere(bad)[:4], got[bad][:4], ref[bad][:4])


def values(q, exps, K):
    return R.fp4_values(R.fp4_codes(q.cpu().numpy(), K), exps.cpu().numpy())


def wide_rows(N, K, seed, dtype):
    """Rows whose groups span many scales, ties and group maxima at the borders among them."""
    x = rows(N, K, seed, "float32").numpy()
    r = np.random.default_rng(seed)
    x *= 2.0 ** r.integers(-12, 13, (N, 1))
    ties = r.choice([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0, 6.0, 0.0], (N, K)) * r.choice([-1, 1], (N, K))
    x = np.where(r.random((N, 1)) < 0.3, ties, x)
    return torch.from_numpy(x.astype(np.float32)).to(DTYPES[dtype])


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("N,K", SHAPES)
def test_pack_and_unpack(cuda_device, N, K, dtype):
    x = wide_rows(N, K, N + K, dtype)
    q, exps = B.fp4_pack(x.to(cuda_device))
    code, ref = R.fp4_pack(f64(x))
    assert np.array_equal(exps.cpu().numpy(), ref)
    want = R.fp4_values(code, ref)
    same(values(q, exps, K), want)
    for out in DTYPES:
        v = B.fp4_unpack(q, exps, K, DTYPES[out])
        exact = torch.from_numpy(want).to(DTYPES[out])
        same(v, exact.double().numpy())


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("pad,offset", [(0, 0), (1, 1), (3, 2), (8, 8), (5, 4)])
@pytest.mark.parametrize("K", [64, 98, 203, 1024])
def test_pack_strides(cuda_device, K, pad, offset, dtype):
    """Rows of other strides and alignments, in and out; nothing outside the rows is written, and the
    codes past K and the bytes past the last group are 0."""
    N = 35
    x = wide_rows(N, K, K, dtype)
    X, _ = strided(x, pad, offset, cuda_device)
    G = (K + 31) // 32
    ke = (G + 3) // 4 * 4
    qb = torch.full((N + 1, G * 16 + 16), 99, dtype=torch.uint8, device=cuda_device)
    eb = torch.full((N + 1, ke + 4), 99, dtype=torch.uint8, device=cuda_device)
    q, exps = qb[:N, :(K + 1) // 2], eb[:N, :G]
    B.bigcn_fp4_pack(X, q, exps)
    code, ref = R.fp4_pack(f64(x))
    same(values(q, exps, K), R.fp4_values(code, ref))
    assert np.array_equal(exps.cpu().numpy(), ref)
    assert (R.fp4_codes(qb[:N, :G * 16].cpu().numpy(), G * 32)[:, K:] == 0).all()
    assert (qb[:N, G * 16:] == 99).all() and (qb[N] == 99).all()
    assert (eb[:N, G:ke] == 0).all() and (eb[:N, ke:] == 99).all() and (eb[N] == 99).all()
    Y, buf = strided(torch.zeros_like(x), pad, offset, cuda_device, fill=7.0)
    B.bigcn_fp4_unpack(q, exps, Y)
    same(Y, torch.from_numpy(R.fp4_values(code, ref)).to(DTYPES[dtype]).double().numpy())
    Y.fill_(7.0)
    assert (buf == 7.0).all()


def test_special_groups(cuda_device):
    """NaN, infinities, zeros, subnormals, the largest values; each in its own group only."""
    x = np.ones((9, 96), np.float32)
    x[0, 40] = np.nan
    x[1, 95] = -np.inf
    x[2, 32:64] = 0.0
    x[3, 32:64] = 2.0 ** -149
    x[4, 32:64] = 2.0 ** -127
    x[5, 32:64] = np.finfo(np.float32).max
    x[6, 33] = 1.74 * 2.0 ** 127
    x[7, 0:32] = -0.0
    x[8].view(np.uint32)[64] = 0x7F800001         # a NaN whose upper half is an infinity's
    code, ref = R.fp4_pack(x)
    q, exps = B.fp4_pack(torch.from_numpy(x).to(cuda_device))
    assert np.array_equal(exps.cpu().numpy(), ref)
    want = R.fp4_values(code, ref)
    same(values(q, exps, 96), want)
    with np.errstate(over="ignore"):
        same(B.fp4_unpack(q, exps, 96), want.astype(np.float32).astype(np.float64))
    # Bytes that only other programs write: 0 is 2^-127, 254 is 2^127.
    exps[0, 0], exps[1, 0] = 0, 254
    v = B.fp4_unpack(q, exps, 96, torch.float32)
    assert v[0, 0].item() == 4.0 * 2.0 ** -127 and v[1, 0].item() == np.inf


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("K,F", [(1, 1), (33, 5), (64, 64), (203, 19), (1433, 64), (602, 128), (31, 130),
                                 (4100, 3), (256, 33), (7, 70001)])
def test_pack_columns(cuda_device, K, F, dtype):
    w = wide_rows(K, F, K + F, dtype)
    q, exps = B.fp4_pack_columns(w.to(cuda_device))
    code, ref = R.fp4_pack(f64(w).T)
    assert np.array_equal(exps.cpu().numpy(), ref)
    same(values(q, exps, K), R.fp4_values(code, ref))
    if F <= 200:
        W, _ = strided(w, 3, 1, cuda_device)
        G = (K + 31) // 32
        ke = (G + 3) // 4 * 4
        qb = torch.full((F + 1, G * 16 + 32), 99, dtype=torch.uint8, device=cuda_device)
        eb = torch.full((F + 1, ke + 4), 99, dtype=torch.uint8, device=cuda_device)
        B.bigcn_fp4_pack_columns(W, qb[:F, :(K + 1) // 2], eb[:F, :G])
        same(values(qb[:F, :(K + 1) // 2], eb[:F, :G], K), R.fp4_values(code, ref))
        assert (R.fp4_codes(qb[:F, :G * 16].cpu().numpy(), G * 32)[:, K:] == 0).all()
        assert (qb[:F, G * 16:] == 99).all() and (qb[F] == 99).all()
        assert (eb[:F, G:ke] == 0).all() and (eb[:F, ke:] == 99).all() and (eb[F] == 99).all()


GEMM = [(1, 1, 1), (1, 203, 64), (2, 32, 7), (5, 33, 33), (127, 64, 32), (129, 96, 40), (128, 128, 128),
        (300, 602, 128), (77, 1433, 64), (1000, 128, 602), (33, 4100, 65), (520, 256, 300), (1, 8192, 1024),
        (260, 2050, 256), (20000, 70, 9), (40000, 200, 200), (7, 32768, 5), (19500, 320, 256)]


def operands(N, K, F, device, seed=0):
    a, b = wide_rows(N, K, N + K + seed, "float32"), rows(F, K, F + K + seed, "float32")
    qa, qb = B.fp4_pack(a.to(device)), B.fp4_pack(b.to(device))
    return qa, qb, values(*qa, K), values(*qb, K)


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("N,K,F", GEMM)
def test_gemm(cuda_device, N, K, F, dtype):
    qa, qb, a, b = operands(N, K, F, cuda_device)
    if dtype == "float16":          # within its range
        qa = B.fp4_pack(torch.from_numpy(rows(N, K, 5, "float32").numpy()).to(cuda_device))
        a = values(*qa, K)
    bias = rows(1, F, 9, "float32")[0]
    for with_bias in (False, True):
        Z = B.fp4_gemm(*qa, *qb, K, bias.to(cuda_device) if with_bias else None, DTYPES[dtype])
        c = f64(bias) if with_bias else 0.0
        within(Z, R.fp4_gemm(a, b, c), R.fp4_gemm_bounds(a, b, c, dtype), "Z")
    assert B.device_timeouts() == 0


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("pad,offset", [(1, 1), (2, 2), (3, 0), (8, 4), (16, 3)])
@pytest.mark.parametrize("N,K,F", [(35, 98, 37), (300, 256, 200), (130, 602, 64)])
def test_gemm_strides(cuda_device, N, K, F, pad, offset, dtype):
    """Operand rows with junk behind them (not in the codes past K), Z's rows of any stride and
    alignment; nothing outside Z's rows is written."""
    (q0, e0), (q1, e1), a, b = operands(N, K, F, cuda_device)
    a, b = a / 64, b / 8
    G = (K + 31) // 32
    ke = (G + 3) // 4 * 4

    def junk(q, e, rows, shift):
        qb = torch.full((rows, G * 16 + 32), 0xFF, dtype=torch.uint8, device=cuda_device)
        eb = torch.full((rows, ke + 8), 0xFF, dtype=torch.uint8, device=cuda_device)
        qb[:, :G * 16] = 0
        qb[:, :(K + 1) // 2] = q
        eb[:, :G] = (e.int() - shift).to(torch.uint8)
        return qb[:, :(K + 1) // 2], eb[:, :G]

    Z, buf = strided(torch.zeros(N, F, dtype=DTYPES[dtype]), pad, offset, cuda_device, fill=7.0)
    B.bigcn_fp4_gemm(*junk(q0, e0, N, 6), *junk(q1, e1, F, 3), K, Z)
    within(Z, R.fp4_gemm(a, b, 0.0), R.fp4_gemm_bounds(a, b, 0.0, dtype), "Z")
    Z.fill_(7.0)
    assert (buf == 7.0).all()


def test_gemm_special_groups(cuda_device):
    """A group of NaN reaches the sums that it is part of and no others; scales from the least to the
    largest; bytes 0 and 254."""
    N, K, F = 140, 160, 70
    (qa, ea), (qb, eb), _, _ = operands(N, K, F, cuda_device)
    ea[3, 2], eb[66, 4], qa[3, 32:48], qb[66, 64:80] = 255, 255, 0, 0
    ea[7], ea[8], eb[9, 0] = 1, 0, 254
    ea[9] = 0
    a, b = values(qa, ea, K), values(qb, eb, K)
    Z = f64(B.fp4_gemm(qa, ea, qb, eb, K))
    ref = R.fp4_gemm(np.nan_to_num(a), np.nan_to_num(b), 0.0)
    bound = R.fp4_gemm_bounds(np.nan_to_num(a), np.nan_to_num(b), 0.0, "float32") + 2.0 ** -126
    nan = np.zeros((N, F), bool)
    nan[3], nan[:, 66] = True, True
    assert np.array_equal(np.isnan(Z), nan)
    # Sums past fp32's range (column 9's, with a scale of 2^127) are infinities.
    past = np.abs(ref) > np.finfo(np.float32).max
    assert past[:, [j for j in range(F) if j != 9]].sum() == 0
    assert np.array_equal(Z[past & ~nan], np.sign(ref[past & ~nan]) * np.inf)
    out = nan | past
    within(np.where(out, 0.0, Z), np.where(out, 0.0, ref), bound, "Z")


@pytest.mark.parametrize("K,F", [(1000, 300), (4100, 256)])
def test_gemm_rows_do_not_depend_on_others(cuda_device, K, F):
    """A row's products are the same bits alone, among others, and in another tile of columns."""
    (qa, ea), (qb, eb), _, _ = operands(2000, K, F, cuda_device)
    Z = B.fp4_gemm(qa, ea, qb, eb, K)
    for i in (0, 127, 128, 1999):
        assert torch.equal(B.fp4_gemm(qa[i:i + 1], ea[i:i + 1], qb, eb, K), Z[i:i + 1])
    assert torch.equal(B.fp4_gemm(qa, ea, qb[64:], eb[64:], K), Z[:, 64:])
    assert torch.equal(B.fp4_gemm(qa, ea, qb[:20], eb[:20], K), Z[:, :20])


def test_two_streams_and_capture(cuda_device):
    """Calls at once on two streams (each takes all tensor memory of its SMs in turn), and a captured
    call replayed on new operands."""
    K, F = 602, 128
    sets = [operands(9000, K, F, cuda_device, seed=s)[:2] for s in (0, 1)]
    want = [B.fp4_gemm(*a, *b, K) for a, b in sets]
    outs = [torch.empty_like(want[0]) for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(20):
        for (a, b), Z, s in zip(sets, outs, streams):
            B.bigcn_fp4_gemm(*a, *b, K, Z, stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, outs))
    X = rows(500, K, 3, "float32").to(cuda_device)
    a, Z = B.fp4_pack(X), torch.empty((500, F), device=cuda_device)
    b = sets[0][1]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        B.bigcn_fp4_pack(X, *a)
        B.bigcn_fp4_gemm(*a, *b, K, Z)
    X.mul_(-3.0)
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(Z, B.fp4_gemm(*B.fp4_pack(X), *b, K))
    assert B.device_timeouts() == 0


def test_no_rows(cuda_device):
    q, e = B.fp4_pack(torch.empty((0, 70), device=cuda_device))
    assert B.fp4_unpack(q, e, 70).shape == (0, 70)
    b = B.fp4_pack(torch.ones((3, 70), device=cuda_device))
    assert B.fp4_gemm(q, e, *b, 70).shape == (0, 3)
