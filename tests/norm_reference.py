"""Layer norm, 8-bit checkpoints and the weight gradient behind them in 64 bits (numpy), and
the error bounds of fp32 evaluations.

Bounds. u = 2^-24 is fp32's unit roundoff. A sum of n terms in which a term passes through at
most D additions is within D u sum |terms| of the exact one. Row sums: a thread of a row's 32
or more adds at most K / 32 terms, then come at most 5 + 32 more: D <= K / 32 + 40. Sums over
rows: at most 1024 runs of rows, each itself of no more additions than N / 8: D <= min(N, 1024)
+ N / 8 + 40 (an order on the tensor cores may truncate instead of rounding: 2 u an addition).
"""
import numpy as np

U = 2.0 ** -24
OUT_ROUND = {"float32": (0.0, 0.0), "bfloat16": (2.0 ** -8, 2.0 ** -134),
             "float16": (2.0 ** -11, 2.0 ** -25)}     # half an ulp: relative, subnormal
GROUP = 32


def row_depth(K):
    return K / 32 + 40


def column_depth(N):
    return min(N, 1024) + N / 8 + 40


# -------------------------------------------------------------- checkpoint ----
def pack(x):
    """(q int8, exps uint8) of fp32-representable rows."""
    x = np.asarray(x, np.float64)
    N, K = x.shape
    G = -(-K // GROUP)
    q, exps = np.zeros((N, K), np.int8), np.zeros((N, G), np.uint8)
    for g in range(G):
        v = x[:, g * GROUP:(g + 1) * GROUP]
        for i in range(N):
            if not np.isfinite(v[i]).all():
                exps[i, g] = 255
                continue
            e = -126
            top = np.abs(v[i]).max()
            while np.rint(top / 2.0 ** e) > 127:
                e += 1
            exps[i, g] = e + 127
            q[i, g * GROUP:(g + 1) * GROUP] = np.rint(v[i] / 2.0 ** e)
    return q, exps


def values(q, exps):
    step = np.where(exps == 255, np.nan, 2.0 ** (exps.astype(np.float64) - 127))
    return q.astype(np.float64) * np.repeat(step, GROUP, axis=1)[:, :q.shape[1]]


# -------------------------------------------------------------- layer norm ----
def forward(x, gamma, beta, eps):
    x = np.asarray(x, np.float64)
    mean = x.mean(1)
    rstd = 1.0 / np.sqrt(((x - mean[:, None]) ** 2).mean(1) + eps)
    xhat = (x - mean[:, None]) * rstd[:, None]
    return xhat * gamma + beta, mean, rstd, xhat


def forward_bounds(x, gamma, beta, eps, dtype):
    """Bounds of |y|, |mean|, |rstd| and |xhat| errors."""
    x = np.asarray(x, np.float64)
    K = x.shape[1]
    y, mean, rstd, xhat = forward(x, gamma, beta, eps)
    D = row_depth(K)
    em = (D + 2) * U * np.abs(x).mean(1)
    # The variance: terms (x - mean)^2 of relative error 3u, D additions; the error of the
    # mean adds its square (the cross term's sum is the deviations', 0).
    var = ((x - mean[:, None]) ** 2).mean(1)
    ev = (D + 6) * U * var + 4 * em ** 2 + 2 * em * U * np.abs(x).mean(1)
    er = rstd * (0.5 * ev / (var + eps) + 4 * U)
    ex = (em[:, None] + U * np.abs(x - mean[:, None])) * rstd[:, None] + \
        np.abs(x - mean[:, None]) * er[:, None] + 2 * U * np.abs(xhat)
    r, a = OUT_ROUND[dtype]
    ey = np.abs(gamma) * ex + 2 * U * (np.abs(gamma * xhat) + np.abs(beta))
    ey = ey + r * (np.abs(y) + ey) + a
    return ey, em, er, ex


def backward(dy, gamma, xhat, rstd):
    g = dy * gamma
    c0, c1 = g.mean(1, keepdims=True), (g * xhat).mean(1, keepdims=True)
    return (g - c0 - xhat * c1) * rstd[:, None], (dy * xhat).sum(0), dy.sum(0)


def backward_bounds(dy, gamma, xhat, rstd, dtype, xhat_error):
    """xhat_error: the error of the xhat that the kernel forms (0 from a checkpoint)."""
    N, K = dy.shape
    g = dy * gamma
    D = row_depth(K)
    e0 = (D + 2) * U * np.abs(g).mean(1)
    e1 = (D + 4) * U * np.abs(g * xhat).mean(1) + (np.abs(g) * xhat_error).mean(1)
    c0, c1 = np.abs(g.mean(1)), np.abs((g * xhat).mean(1))
    e = e0[:, None] + np.abs(xhat) * e1[:, None] + xhat_error * c1[:, None] + \
        5 * U * (np.abs(g) + c0[:, None] + np.abs(xhat) * c1[:, None])
    dx = backward(dy, gamma, xhat, rstd)[0]
    r, a = OUT_ROUND[dtype]
    e = e * rstd[:, None] + 2 * U * np.abs(dx)
    e = e + r * (np.abs(dx) + e) + a
    Dn = column_depth(N)
    eg = (Dn + 2) * U * np.abs(dy * xhat).sum(0) + (np.abs(dy) * xhat_error).sum(0)
    return e, eg, Dn * U * np.abs(dy).sum(0)


# --------------------------------------------------- the product's gradients ----
def weight_grad(v, gamma, beta, dz):
    db = dz.sum(0)
    return gamma[:, None] * (v.T @ dz) + beta[:, None] * db, db


def weight_grad_bounds(v, gamma, beta, dz):
    N = dz.shape[0]
    D = 2 * column_depth(N) + 4
    s = np.abs(v).T @ np.abs(dz)
    b = np.abs(dz).sum(0)
    return (D * U * (np.abs(gamma)[:, None] * s + np.abs(beta)[:, None] * b), D * U * b)
