"""Argument checks of the residual layer's operators, without a GPU: each refusal comes before any
CUDA call (fake, never-dereferenced pointers are enough)."""
import ctypes

import pytest
import torch

from paper_2010_07565_gb300 import build as lib_build

OK, INVALID, MISALIGNED = 0, 1, 2
P = 1 << 32
STEP = 1 << 24
F32, BF16, F16 = 0, 1, 2


@pytest.fixture(scope="module")
def lib():
    from paper_2010_07565_gb300 import binding
    lib_build.build()
    return binding.lib()


def ptr(n):
    return P + n * STEP


def caller(fn, defaults):
    def call(**kw):
        unknown = set(kw) - set(defaults)
        assert not unknown, unknown
        return fn(*{**defaults, **kw}.values(), None)
    return call


def test_rms_norm_forward_refusals(lib):
    f = caller(lib.bigcn_rms_norm_forward, dict(
        dtype=F32, X=ptr(0), N=10, K=70, ldx=70, R=ptr(1), ldr=70, gamma=ptr(2), eps=1e-5, S=ptr(3),
        lds=70, Y=ptr(4), ldy=70, rstd=ptr(5), q=ptr(6), ldq=80, exps=ptr(7), lde=4))
    assert f(N=0) == OK
    assert f(N=0, S=ptr(1)) == OK and f(N=0, R=None, S=None) == OK
    for kw in (dict(dtype=3), dict(N=-1), dict(N=1 << 31), dict(K=0), dict(K=(1 << 30) + 1), dict(ldx=69),
               dict(ldr=69), dict(lds=69), dict(ldy=69), dict(eps=-1e-9), dict(eps=float("nan")),
               dict(eps=float("inf")), dict(q=None), dict(exps=None), dict(X=None), dict(R=None),
               dict(ldq=72), dict(lde=3), dict(lde=6), dict(ldx=1 << 60), dict(ldr=1 << 60),
               dict(S=None, Y=None, rstd=None, q=None, exps=None),
               dict(Y=ptr(0)), dict(Y=ptr(1)), dict(Y=ptr(3)), dict(S=ptr(0) + 4), dict(S=ptr(1) + 280),
               dict(S=ptr(1), lds=71), dict(S=ptr(0), lds=80), dict(rstd=ptr(2)), dict(q=ptr(4)),
               dict(exps=ptr(6) + 16), dict(rstd=ptr(5), Y=ptr(5) + 4), dict(S=ptr(1), Y=ptr(1))):
        assert f(**kw) == INVALID, kw
    for kw in (dict(X=ptr(0) + 2), dict(R=ptr(1) + 1), dict(S=ptr(3) + 2), dict(Y=ptr(4) + 3),
               dict(gamma=ptr(2) + 2), dict(rstd=ptr(5) + 1), dict(q=ptr(6) + 8),
               dict(exps=ptr(7) + 2), dict(dtype=F16, X=ptr(0) + 1)):
        assert f(**kw) == MISALIGNED, kw


def test_rms_norm_backward_workspace(lib):
    f = lib.bigcn_rms_norm_backward_workspace_bytes
    assert f(0, 5) == 256 and f(7, 100) == 2816 and f(1 << 20, 64) == 1024 * 256
    assert f(-1, 5) == 0 and f(5, 0) == 0 and f(5, (1 << 30) + 1) == 0 and f(1 << 31, 4) == 0


def test_rms_norm_backward_refusals(lib):
    kept = dict(S=None, q=ptr(3), exps=ptr(4))
    f = caller(lib.bigcn_rms_norm_backward, dict(
        dtype=F32, dY=ptr(0), N=10, K=70, lddy=70, gamma=ptr(1), S=ptr(2), lds=70, q=None, ldq=80,
        exps=None, lde=4, rstd=ptr(5), dS=ptr(6), ldds=70, dX=ptr(7), lddx=70, dgamma=ptr(8),
        workspace=ptr(9), ws=lib.bigcn_rms_norm_backward_workspace_bytes(10, 70)))
    assert f(N=0, dgamma=None) == OK and f(N=0, dgamma=None, **kept) == OK
    for kw in (dict(dtype=-1), dict(N=-1), dict(N=1 << 31), dict(K=0), dict(lddy=69), dict(lds=69),
               dict(ldds=69), dict(lddx=69), dict(dX=None), dict(dX=None, dS=None, dgamma=None),
               dict(S=None), dict(q=ptr(3), exps=ptr(4)), dict(S=None, q=ptr(3)),
               dict(S=None, exps=ptr(4)), dict(dY=None), dict(rstd=None), dict(workspace=None),
               dict(ws=100), dict(lddy=1 << 60), dict(ldds=1 << 60),
               dict(kept, ldq=72), dict(kept, lde=3), dict(dX=ptr(0)), dict(dX=ptr(2)),
               dict(dX=ptr(6) + 4), dict(dX=ptr(6), lddx=71), dict(dgamma=ptr(1)),
               dict(dgamma=ptr(6)), dict(workspace=ptr(6)), dict(workspace=ptr(7)),
               dict(kept, dX=ptr(3)), dict(kept, dgamma=ptr(4))):
        assert f(**kw) == INVALID, kw
    for kw in (dict(dY=ptr(0) + 2), dict(gamma=ptr(1) + 2), dict(S=ptr(2) + 1), dict(rstd=ptr(5) + 2),
               dict(dS=ptr(6) + 2), dict(dX=ptr(7) + 2), dict(dgamma=ptr(8) + 2),
               dict(workspace=ptr(9) + 128), dict(kept, q=ptr(3) + 8), dict(kept, exps=ptr(4) + 1)):
        assert f(**kw) == MISALIGNED, kw


@pytest.mark.parametrize("columns", [False, True])
def test_fp4_pack_refusals(lib, columns):
    if columns:
        f = caller(lib.bigcn_fp4_pack_columns, dict(dtype=F32, X=ptr(0), K=70, N=10, ldx=10, q=ptr(1),
                                                    ldq=48, exps=ptr(2), lde=4))
        bad = [dict(N=0), dict(ldx=9), dict(N=(1 << 30) + 1)]
    else:
        f = caller(lib.bigcn_fp4_pack, dict(dtype=F32, X=ptr(0), N=10, K=70, ldx=70, q=ptr(1), ldq=48,
                                            exps=ptr(2), lde=4))
        bad = [dict(N=1 << 31), dict(ldx=69)]
        assert f(N=0) == OK
    for kw in bad + [dict(dtype=3), dict(N=-1), dict(K=0), dict(K=(1 << 30) + 1), dict(ldq=32),
                     dict(ldq=56), dict(lde=2), dict(lde=6), dict(X=None), dict(q=None),
                     dict(exps=None), dict(q=ptr(0)), dict(exps=ptr(1) + 16), dict(exps=ptr(0) + 4),
                     dict(ldx=1 << 60), dict(ldq=1 << 60)]:
        assert f(**kw) == INVALID, kw
    for kw in (dict(X=ptr(0) + 2), dict(q=ptr(1) + 8), dict(exps=ptr(2) + 2),
               dict(dtype=BF16, X=ptr(0) + 1)):
        assert f(**kw) == MISALIGNED, kw


def test_fp4_unpack_refusals(lib):
    f = caller(lib.bigcn_fp4_unpack, dict(dtype=F32, q=ptr(1), ldq=48, exps=ptr(2), lde=4, N=10, K=70,
                                          X=ptr(0), ldx=70))
    assert f(N=0) == OK
    for kw in (dict(dtype=7), dict(N=-1), dict(K=0), dict(ldx=69), dict(ldq=32), dict(lde=5),
               dict(q=None), dict(exps=None), dict(X=None), dict(X=ptr(1)), dict(X=ptr(2))):
        assert f(**kw) == INVALID, kw
    for kw in (dict(X=ptr(0) + 1), dict(q=ptr(1) + 4), dict(exps=ptr(2) + 1)):
        assert f(**kw) == MISALIGNED, kw


def test_fp4_gemm_refusals(lib):
    f = caller(lib.bigcn_fp4_gemm, dict(
        dtype=F32, aq=ptr(0), ldaq=48, ae=ptr(1), ldae=4, N=10, bq=ptr(2), ldbq=48, be=ptr(3), ldbe=4,
        F=7, K=70, bias=ptr(4), Z=ptr(5), ldz=7))
    assert f(N=0) == OK
    for kw in (dict(dtype=3), dict(N=-1), dict(N=1 << 31), dict(K=0), dict(K=32769, ldaq=1 << 15,
               ldbq=1 << 15, ldae=2048, ldbe=2048), dict(F=0), dict(F=(1 << 30) + 1), dict(ldz=6),
               dict(ldaq=32), dict(ldbq=40), dict(ldae=2), dict(ldbe=6), dict(aq=None), dict(ae=None),
               dict(bq=None), dict(be=None), dict(Z=None), dict(Z=ptr(0)), dict(Z=ptr(1)),
               dict(Z=ptr(2)), dict(Z=ptr(3)), dict(Z=ptr(4)), dict(ldz=1 << 60), dict(ldaq=1 << 60)):
        assert f(**kw) == INVALID, kw
    for kw in (dict(aq=ptr(0) + 8), dict(ae=ptr(1) + 2), dict(bq=ptr(2) + 4), dict(be=ptr(3) + 1),
               dict(Z=ptr(5) + 2), dict(bias=ptr(4) + 2), dict(dtype=BF16, Z=ptr(5) + 1)):
        assert f(**kw) == MISALIGNED, kw


def clip_args(lib, ts, out, **kw):
    """ts, out: (dtype, pointer, count) and pointers."""
    n = len(ts)
    d = dict(n=n, dtypes=(ctypes.c_int32 * n)(*[t[0] for t in ts]),
             tensors=(ctypes.c_void_p * n)(*[t[1] for t in ts]),
             out=(ctypes.c_void_p * n)(*out) if out is not None else None,
             counts=(ctypes.c_int64 * n)(*[t[2] for t in ts]), max_norm=1.0, norm=ptr(100),
             ws=ptr(101), bytes=lib.bigcn_grad_norm_workspace_bytes(n))
    return {**d, **kw}


def test_grad_norm_refusals(lib):
    def norm(ts, **kw):
        d = clip_args(lib, ts, None, **kw)
        return lib.bigcn_grad_norm(*[d[k] for k in ("n", "dtypes", "tensors", "counts", "norm", "ws",
                                                    "bytes")], None)

    def clip(ts, out=None, **kw):
        d = clip_args(lib, ts, [t[1] for t in ts] if out is None else out, **kw)
        return lib.bigcn_clip_grad_norm(*d.values(), None)

    good = [(F32, ptr(0), 100), (BF16, ptr(1), 7), (F16, None, 0)]
    for f in (norm, clip):
        for kw in (dict(n=-1), dict(n=65537), dict(norm=None), dict(ws=None), dict(bytes=8),
                   dict(dtypes=None), dict(tensors=None), dict(counts=None), dict(ws=ptr(0) - 256),
                   dict(norm=ptr(1)), dict(norm=ptr(101) + 4)):
            assert f(good, **kw) == INVALID, kw
        for bad in ((3, ptr(2), 5), (F32, None, 5), (F32, ptr(2), -1), (F32, ptr(2), 1 << 61)):
            assert f(good + [bad]) == INVALID, bad
        for bad in ((F32, ptr(2) + 2, 5), (F16, ptr(2) + 1, 5)):
            assert f(good + [bad]) == MISALIGNED, bad
        assert f(good, norm=ptr(100) + 2) == MISALIGNED
        assert f(good, ws=ptr(101) + 8) == MISALIGNED
    # A tensor twice, or overlapping ones: never to scale.
    assert clip(good + [(F32, ptr(0), 100)]) == INVALID
    assert clip(good + [(BF16, ptr(0) + 398, 9)]) == INVALID
    out = [ptr(10), ptr(11), None]
    assert clip(good, [ptr(10), ptr(10) + 64, None]) == INVALID
    assert clip(good, [ptr(1), ptr(11), None]) == INVALID          # one tensor's place is another's out
    assert clip(good, [ptr(0) + 4, ptr(11), None]) == INVALID      # in place, but not quite
    assert clip(good, [None, ptr(11), None]) == INVALID
    assert clip(good, [ptr(10) + 2, ptr(11), None]) == MISALIGNED
    assert clip(good, [ptr(10), ptr(101) + 8, None]) == INVALID
    for m in (-1.0, float("nan")):
        assert clip(good, out, max_norm=m) == INVALID


def test_binding_refuses_wrong_tensors(lib):
    """Types, shapes and tensors that are not on the device, before anything is called."""
    from paper_2010_07565_gb300 import binding as B
    z = torch.zeros
    q, e = B.fp4_buffers(4, 70, "cpu")
    assert q.shape == (4, 35) and q.stride(0) == 48 and e.shape == (4, 3) and e.stride(0) == 4
    X, g = z(4, 70), z(70)
    for call in (
            lambda: B.bigcn_rms_norm_forward(X, g, 1e-5, R=z(4, 71), Y=z(4, 70)),
            lambda: B.bigcn_rms_norm_forward(X, g, 1e-5, R=z(4, 70).half(), Y=z(4, 70)),
            lambda: B.bigcn_rms_norm_forward(X, z(71), 1e-5, Y=z(4, 70)),
            lambda: B.bigcn_rms_norm_forward(X.double(), g, 1e-5, Y=z(4, 70).double()),
            lambda: B.bigcn_rms_norm_forward(X, g, 1e-5, Y=z(70, 4).t()),
            lambda: B.bigcn_rms_norm_forward(X, g, 1e-5, Y=z(4, 70)),
            lambda: B.bigcn_rms_norm_backward(X, g, z(4), z(256), S=z(4, 71), dX=z(4, 70)),
            lambda: B.bigcn_rms_norm_backward(X, g, z(3), z(256), S=z(4, 70), dX=z(4, 70)),
            lambda: B.bigcn_rms_norm_backward(X, g, z(4), None, S=z(4, 70), dX=z(4, 70)),
            lambda: B.bigcn_fp4_pack(X, q[:, :34], e),
            lambda: B.bigcn_fp4_pack(X, q.to(torch.int8), e),
            lambda: B.bigcn_fp4_pack(X, q, e),
            lambda: B.bigcn_fp4_unpack(q, e, X),
            lambda: B.bigcn_fp4_pack_columns(z(70, 5), q, e),
            lambda: B.bigcn_fp4_pack_columns(z(70, 4), q, e),
            lambda: B.bigcn_fp4_gemm(q, e, q, e, 70, z(4, 5)),
            lambda: B.bigcn_fp4_gemm(q, e, q, e, 72, z(4, 4)),
            lambda: B.bigcn_fp4_gemm(q, e, q, e, 70, z(4, 4), bias=z(4).half()),
            lambda: B.bigcn_fp4_gemm(q, e, q, e, 70, z(4, 4)),
            lambda: B.TensorList([z(4, 4).t()[:, :2]]),
            lambda: B.TensorList([z(4).long()]),
            lambda: B.bigcn_grad_norm([X], z(2), z(8192)),
            lambda: B.bigcn_grad_norm([X], z(1), z(8192)),
            lambda: B.bigcn_clip_grad_norm([X], 1.0, z(1), z(8192), out=[z(279)]),
            lambda: B.bigcn_clip_grad_norm([X], 1.0, z(1), z(8192), out=[z(4, 70).half()]),
            lambda: B.bigcn_clip_grad_norm([X], 1.0, z(1), z(8192))):
        with pytest.raises(ValueError):
            call()


def test_grad_norm_workspace(lib):
    f = lib.bigcn_grad_norm_workspace_bytes
    assert f(-1) == 0 and f(65537) == 0 and f(0) >= 8 and f(65536) % 256 == 0
    assert f(1) >= f(0) and f(65536) > f(1)
