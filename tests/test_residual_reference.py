"""The 64-bit forms of the residual layer's operators against forms written another way (no GPU)."""
import numpy as np
import pytest

import residual_reference as R


def test_rms_backward_follows_differences():
    r = np.random.default_rng(1)
    N, K, h = 3, 7, 1e-6
    s, gamma, dy, ds = r.standard_normal((N, K)), r.standard_normal(K), *r.standard_normal((2, N, K))
    _, rstd, shat = R.rms_forward(s, gamma, 1e-3)
    dx, dg = R.rms_backward(dy, gamma, shat, rstd, ds)
    loss = lambda s, g: (R.rms_forward(s, g, 1e-3)[0] * dy + s * ds).sum()
    for i in range(N):
        for k in range(K):
            d = np.zeros((N, K))
            d[i, k] = h
            assert abs((loss(s + d, gamma) - loss(s - d, gamma)) / (2 * h) - dx[i, k]) < 1e-8
    for k in range(K):
        d = np.zeros(K)
        d[k] = h
        assert abs((loss(s, gamma + d) - loss(s, gamma - d)) / (2 * h) - dg[k]) < 1e-8


def test_fp4_ties_go_to_the_even_code():
    m = [0, 0.25, 0.26, 0.75, 0.74, 1.25, 1.3, 1.75, 1.7, 2.5, 2.6, 3.5, 3.4, 5.0, 5.1, 6.9]
    assert R.fp4_nearest(m).tolist() == [0, 0, 1, 2, 1, 2, 3, 4, 3, 4, 5, 6, 5, 6, 7, 7]


@pytest.mark.parametrize("top,byte", [(6.0, 127), (6.99, 127), (7.0, 128), (4.0, 127), (3.99, 127),
                                      (3.5, 127), (3.49, 126), (0.0, 1), (2.0 ** -140, 1), (3.4e38, 253),
                                      (2.0 ** 127, 252)])
def test_fp4_scale_byte_is_the_least_that_fits(top, byte):
    x = np.zeros((1, 40))
    x[0, 35] = -top
    code, exps = R.fp4_pack(x)
    assert exps.tolist() == [[1, byte]]
    v = R.fp4_values(code, exps)
    assert abs(v[0, 35] + top) <= max(top / 5, 2.0 ** (int(byte) - 127) / 4)


def test_fp4_bad_groups_are_nan():
    x = np.ones((2, 64))
    x[0, 40], x[1, 3] = np.nan, -np.inf
    v = R.fp4_values(*R.fp4_pack(x))
    assert np.isnan(v).tolist() == [[False] * 32 + [True] * 32, [True] * 32 + [False] * 32]


def test_clip_leaves_small_norms():
    t = [np.array([3.0, 0.0]), np.array([4.0])]
    norm, out = R.clip(t, 10.0)
    assert norm == 5.0 and all(np.array_equal(a, b) for a, b in zip(t, out))
    norm, out = R.clip(t, 1.0)
    assert np.allclose(np.concatenate(out), [0.6, 0.0, 0.8], rtol=1e-15)
