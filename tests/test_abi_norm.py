"""Argument checks of layer norm, the checkpoints and the weight gradient, without a GPU: each
refusal comes before any CUDA call (fake, never-dereferenced pointers are enough)."""
import pytest

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


def test_checkpoint_groups(lib):
    assert [lib.bigcn_checkpoint_groups(k) for k in (-1, 0, 1, 32, 33, 64, 65)] == \
        [0, 0, 1, 1, 2, 2, 3]


def pack_args(**kw):
    d = dict(dtype=F32, X=ptr(0), N=10, K=70, ldx=70, q=ptr(1), ldq=80, exps=ptr(2), lde=4)
    d.update(kw)
    return [d[k] for k in ("dtype", "X", "N", "K", "ldx", "q", "ldq", "exps", "lde")] + [None]


def test_checkpoint_pack_refusals(lib):
    f = lambda **kw: lib.bigcn_checkpoint_pack(*pack_args(**kw))
    assert f(N=0) == OK
    for kw in (dict(dtype=3), dict(dtype=-1), dict(N=-1), dict(N=1 << 31), dict(K=0), dict(ldx=69),
               dict(ldq=72), dict(ldq=64), dict(lde=3), dict(lde=6), dict(X=None), dict(q=None),
               dict(exps=None), dict(q=ptr(0)), dict(exps=ptr(1) + 16), dict(ldx=1 << 60),
               dict(ldq=1 << 60), dict(exps=ptr(0) + 4)):
        assert f(**kw) == INVALID, kw
    for kw in (dict(X=ptr(0) + 2), dict(q=ptr(1) + 8), dict(exps=ptr(2) + 2),
               dict(dtype=F16, X=ptr(0) + 1)):
        assert f(**kw) == MISALIGNED, kw


def unpack_args(**kw):
    d = dict(dtype=F32, q=ptr(1), ldq=80, exps=ptr(2), lde=4, N=10, K=70, gamma=ptr(3),
             beta=ptr(4), X=ptr(0), ldx=70)
    d.update(kw)
    return [d[k] for k in ("dtype", "q", "ldq", "exps", "lde", "N", "K", "gamma", "beta", "X",
                           "ldx")] + [None]


def test_checkpoint_unpack_refusals(lib):
    f = lambda **kw: lib.bigcn_checkpoint_unpack(*unpack_args(**kw))
    assert f(N=0) == OK
    for kw in (dict(dtype=5), dict(K=0), dict(N=-1), dict(ldx=69), dict(ldq=70), dict(lde=5),
               dict(q=None), dict(exps=None), dict(X=None), dict(X=ptr(1)), dict(X=ptr(3)),
               dict(X=ptr(4) + 40)):
        assert f(**kw) == INVALID, kw
    for kw in (dict(gamma=ptr(3) + 2), dict(beta=ptr(4) + 1), dict(X=ptr(0) + 2),
               dict(q=ptr(1) + 4)):
        assert f(**kw) == MISALIGNED, kw


def forward_args(**kw):
    d = dict(dtype=F32, X=ptr(0), N=10, K=70, ldx=70, gamma=ptr(1), beta=ptr(2), eps=1e-5,
             Y=ptr(3), ldy=70, mean=ptr(4), rstd=ptr(5), q=ptr(6), ldq=80, exps=ptr(7), lde=4)
    d.update(kw)
    return [d[k] for k in ("dtype", "X", "N", "K", "ldx", "gamma", "beta", "eps", "Y", "ldy",
                           "mean", "rstd", "q", "ldq", "exps", "lde")] + [None]


def test_layer_norm_forward_refusals(lib):
    f = lambda **kw: lib.bigcn_layer_norm_forward(*forward_args(**kw))
    assert f(N=0) == OK
    for kw in (dict(dtype=9), dict(N=-1), dict(N=1 << 31), dict(K=0), dict(ldx=69), dict(ldy=69),
               dict(eps=-1e-5), dict(eps=float("nan")), dict(eps=float("inf")), dict(q=None),
               dict(exps=None), dict(ldq=72), dict(lde=2), dict(X=None), dict(Y=None),
               dict(Y=ptr(0)), dict(Y=ptr(0) + 2796), dict(mean=ptr(3)), dict(rstd=ptr(4) + 36),
               dict(q=ptr(3)), dict(exps=ptr(6) + 32), dict(mean=ptr(1) + 4), dict(ldx=1 << 60)):
        assert f(**kw) == INVALID, kw
    for kw in (dict(X=ptr(0) + 2), dict(Y=ptr(3) + 1), dict(gamma=ptr(1) + 2), dict(rstd=ptr(5) + 2),
               dict(q=ptr(6) + 8), dict(exps=ptr(7) + 1)):
        assert f(**kw) == MISALIGNED, kw


def backward_args(lib, **kw):
    N, K = kw.get("N", 10), kw.get("K", 70)
    d = dict(dtype=F32, dY=ptr(0), N=10, K=70, lddy=70, gamma=ptr(1), X=None, ldx=0, mean=None,
             q=ptr(2), ldq=80, exps=ptr(3), lde=4, rstd=ptr(4), dX=ptr(5), lddx=70, dgamma=ptr(6),
             dbeta=ptr(7), ws=ptr(8),
             wsb=lib.bigcn_layer_norm_backward_workspace_bytes(max(N, 0), max(K, 1)))
    d.update(kw)
    return [d[k] for k in ("dtype", "dY", "N", "K", "lddy", "gamma", "X", "ldx", "mean", "q",
                           "ldq", "exps", "lde", "rstd", "dX", "lddx", "dgamma", "dbeta", "ws",
                           "wsb")] + [None]


def test_layer_norm_backward_refusals(lib):
    w = lib.bigcn_layer_norm_backward_workspace_bytes
    assert w(-1, 5) == 0 and w(5, 0) == 0 and w(1 << 31, 5) == 0 and w(100, 70) > 0
    f = lambda **kw: lib.bigcn_layer_norm_backward(*backward_args(lib, **kw))
    need = w(10, 70)
    x = dict(X=ptr(9), ldx=70, mean=ptr(10))
    for kw in (dict(dtype=3), dict(N=-1), dict(K=0), dict(lddy=69), dict(lddx=69),
               dict(dX=None, dgamma=None, dbeta=None),
               x,                                                     # two sources of xhat
               dict(q=None, exps=None), dict(q=None), dict(exps=None),
               dict(x, q=None, exps=None, mean=None), dict(mean=ptr(10)),
               dict(x, q=None, exps=None, ldx=69), dict(ldq=79), dict(lde=3), dict(dY=None),
               dict(rstd=None), dict(ws=None), dict(wsb=need - 1), dict(dX=ptr(0)),
               dict(dX=ptr(2)), dict(dgamma=ptr(1)), dict(dbeta=ptr(6) + 4), dict(ws=ptr(5)),
               dict(dX=ptr(8) + 256), dict(lddy=1 << 60)):
        assert f(**kw) == INVALID, kw
    for kw in (dict(dY=ptr(0) + 2), dict(q=ptr(2) + 1), dict(ws=ptr(8) + 128), dict(dX=ptr(5) + 2),
               dict(dbeta=ptr(7) + 2), dict(rstd=ptr(4) + 2)):
        assert f(**kw) == MISALIGNED, kw


def grad_args(lib, **kw):
    N, K, F = kw.get("N", 100), kw.get("K", 70), kw.get("F", 9)
    d = dict(dtype=F32, q=ptr(0), ldq=80, exps=ptr(1), lde=4, N=100, K=70, gamma=ptr(2),
             beta=ptr(3), dZ=ptr(4), F=9, lddz=9, dW=ptr(5), lddw=9, db=ptr(6), ws=ptr(7),
             wsb=lib.bigcn_checkpoint_weight_grad_workspace_bytes(max(N, 0), max(K, 1), max(F, 1)))
    d.update(kw)
    return [d[k] for k in ("dtype", "q", "ldq", "exps", "lde", "N", "K", "gamma", "beta", "dZ",
                           "F", "lddz", "dW", "lddw", "db", "ws", "wsb")] + [None]


def test_weight_grad_refusals(lib):
    w = lib.bigcn_checkpoint_weight_grad_workspace_bytes
    assert w(-1, 5, 5) == 0 and w(5, 0, 5) == 0 and w(5, 5, 0) == 0 and w(1 << 31, 5, 5) == 0
    assert w(100, 70, 9) > 0
    f = lambda **kw: lib.bigcn_checkpoint_weight_grad(*grad_args(lib, **kw))
    need = w(100, 70, 9)
    for kw in (dict(dtype=4), dict(N=-1), dict(N=1 << 31), dict(K=0), dict(F=0), dict(lddz=8),
               dict(lddw=8), dict(ldq=70), dict(ldq=64), dict(lde=2), dict(q=None),
               dict(exps=None), dict(dZ=None), dict(dW=None), dict(ws=None), dict(wsb=need - 1),
               dict(dW=ptr(0)), dict(dW=ptr(4)), dict(db=ptr(5) + 8), dict(db=ptr(2)),
               dict(ws=ptr(4)), dict(dW=ptr(7) + 256), dict(lddz=1 << 60), dict(lddw=1 << 60)):
        assert f(**kw) == INVALID, kw
    for kw in (dict(q=ptr(0) + 8), dict(exps=ptr(1) + 2), dict(gamma=ptr(2) + 1),
               dict(dZ=ptr(4) + 2), dict(dW=ptr(5) + 2), dict(db=ptr(6) + 2),
               dict(ws=ptr(7) + 64), dict(dtype=BF16, dZ=ptr(4) + 1)):
        assert f(**kw) == MISALIGNED, kw


def test_rows_past_the_widest_are_refused(lib):
    """K and F up to 2^30: the kernels' column indices have 32 bits and step past a row's end."""
    K = (1 << 30) + 16
    wide = dict(K=K, ldx=K, ldq=K, lde=(1 << 25) + 4)
    assert lib.bigcn_checkpoint_pack(*pack_args(X=1 << 40, q=1 << 50, exps=1 << 51, **wide)) == INVALID
    assert lib.bigcn_checkpoint_unpack(*unpack_args(
        X=1 << 40, q=1 << 50, exps=1 << 51, gamma=None, beta=None, **wide)) == INVALID
    assert lib.bigcn_layer_norm_forward(*forward_args(
        X=1 << 40, Y=1 << 45, ldy=K, q=1 << 50, exps=1 << 51, gamma=None, beta=None, **wide)) == INVALID
    assert lib.bigcn_layer_norm_backward_workspace_bytes(10, K) == 0
    assert lib.bigcn_layer_norm_backward(*backward_args(
        lib, K=K, lddy=K, lddx=K, ldq=K, lde=(1 << 25) + 4, dY=1 << 40, dX=1 << 45, q=1 << 50,
        exps=1 << 51, gamma=None, dgamma=None, dbeta=None, ws=None, wsb=0)) == INVALID
    assert lib.bigcn_checkpoint_weight_grad_workspace_bytes(100, K, 9) == 0
    assert lib.bigcn_checkpoint_weight_grad_workspace_bytes(100, 9, K) == 0


def test_backward_workspace_follows_the_rows(lib):
    """A row's sums each, at most 1024 of them: a single wide row needs no more than its own."""
    w = lib.bigcn_layer_norm_backward_workspace_bytes
    assert w(1, 70001) == (2 * 70001 * 4 + 255) // 256 * 256
    assert w(1024, 64) == w(1 << 30, 64) == 1024 * 2 * 64 * 4
    assert 0 < w(0, 64) <= w(1, 64) < w(2, 64)
