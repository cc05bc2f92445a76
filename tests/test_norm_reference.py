"""The 64-bit reference of layer norm, checkpoints and the weight gradient, pinned on the CPU:
gradients against central differences of the forward, the checkpoint against its definition."""
import numpy as np
import pytest

import norm_reference as R


def rng(seed):
    return np.random.Generator(np.random.PCG64(seed))


def test_layer_norm_gradients_match_differences():
    r = rng(1)
    N, K, eps, h = 5, 7, 1e-5, 1e-6
    x, dy = r.standard_normal((N, K)) * 2 + 3, r.standard_normal((N, K))
    gamma, beta = 1 + 0.3 * r.standard_normal(K), r.standard_normal(K)
    loss = lambda x, g, b: (R.forward(x, g, b, eps)[0] * dy).sum()
    _, _, rstd, xhat = R.forward(x, gamma, beta, eps)
    dx, dg, db = R.backward(dy, gamma, xhat, rstd)
    for at in np.ndindex(N, K):
        e = np.zeros((N, K))
        e[at] = h
        d = (loss(x + e, gamma, beta) - loss(x - e, gamma, beta)) / (2 * h)
        assert abs(d - dx[at]) < 1e-7
    for k in range(K):
        e = np.zeros(K)
        e[k] = h
        assert abs((loss(x, gamma + e, beta) - loss(x, gamma - e, beta)) / (2 * h) - dg[k]) < 1e-7
        assert abs((loss(x, gamma, beta + e) - loss(x, gamma, beta - e)) / (2 * h) - db[k]) < 1e-7


def test_weight_gradient_matches_differences():
    r = rng(2)
    N, K, F, h = 6, 5, 3, 1e-6
    v, dz = r.standard_normal((N, K)), r.standard_normal((N, F))
    gamma, beta, W = 1 + r.standard_normal(K), r.standard_normal(K), r.standard_normal((K, F))
    b = r.standard_normal(F)
    loss = lambda W, b: (((gamma * v + beta) @ W + b) * dz).sum()
    dW, db = R.weight_grad(v, gamma, beta, dz)
    for at in np.ndindex(K, F):
        e = np.zeros((K, F))
        e[at] = h
        assert abs((loss(W + e, b) - loss(W - e, b)) / (2 * h) - dW[at]) < 1e-7
    for j in range(F):
        e = np.zeros(F)
        e[j] = h
        assert abs((loss(W, b + e) - loss(W, b - e)) / (2 * h) - db[j]) < 1e-7


@pytest.mark.parametrize("K", [1, 31, 32, 33, 70])
def test_checkpoint_error_and_bytes(K):
    x = rng(K).standard_normal((9, K)).astype(np.float32) * np.float32(10.0) ** np.arange(-4, 5)[:, None]
    q, exps = R.pack(x)
    assert np.abs(q.astype(int)).max() <= 127 and (exps >= 1).all()
    v = R.values(q, exps)
    top = np.stack([np.abs(x[:, g:g + 32]).max(1) for g in range(0, K, 32)], 1)
    assert (np.abs(v - x) <= np.repeat(top, 32, axis=1)[:, :K] * (1 / 127.5) * (1 + 1e-9)).all()
    # The least step: half of it would not hold the largest magnitude.
    assert (np.rint(top / 2.0 ** (exps.astype(float) - 128)) > 127).all()


def test_checkpoint_special_groups():
    x = np.zeros((1, 128), np.float32)
    x[0, 32], x[0, 64], x[0, 96] = 1e-45, np.inf, 127.5
    q, exps = R.pack(x)
    assert list(exps[0]) == [1, 1, 255, 128]         # 127.5 would round to 128: a doubled step
    assert q[0, 96] == 64 and not q[0, :96].any()
    assert np.isnan(R.values(q, exps)[0, 64:96]).all()
