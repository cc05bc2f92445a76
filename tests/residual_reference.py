"""The operators of a residual layer in 64 bits (numpy): root-mean-square norm of a sum, rows in
microscaled 4 bits and their product, the norm of many tensors; and the error bounds of fp32
evaluations (norm_reference has the bounds' terms)."""
import numpy as np

from norm_reference import GROUP, OUT_ROUND, U, column_depth, row_depth


# ---------------------------------------------------------------- rms norm ----
def rms_forward(s, gamma, eps):
    """(Y, rstd, shat) of the rows of s."""
    s = np.asarray(s, np.float64)
    rstd = 1.0 / np.sqrt((s * s).mean(1) + eps)
    shat = s * rstd[:, None]
    return shat * gamma, rstd, shat


def rms_forward_bounds(s, gamma, eps, dtype):
    """Bounds of |Y|, |rstd| and |shat| errors. The mean of squares, all of one sign, is within
    (D + 3) u of itself; the root halves that; root, division and eps's addition round once each."""
    y, rstd, shat = rms_forward(s, gamma, eps)
    er = rstd * (0.5 * (row_depth(s.shape[1]) + 4) + 3) * U
    ex = np.abs(shat) * ((er / rstd)[:, None] + U)
    r, a = OUT_ROUND[dtype]
    ey = np.abs(gamma) * ex + U * np.abs(y)
    return ey + r * (np.abs(y) + ey) + a, er, ex


def rms_backward(dy, gamma, shat, rstd, ds=0.0):
    g = dy * gamma
    c = (g * shat).mean(1, keepdims=True)
    return (g - shat * c) * rstd[:, None] + ds, (dy * shat).sum(0)


def rms_backward_bounds(dy, gamma, shat, rstd, dtype, shat_error, ds=0.0):
    """shat_error: the error of the shat that the kernel forms (0 from a checkpoint)."""
    N, K = dy.shape
    g = dy * gamma
    e1 = (row_depth(K) + 4) * U * np.abs(g * shat).mean(1) + (np.abs(g) * shat_error).mean(1)
    c = np.abs((g * shat).mean(1))
    e = np.abs(shat) * e1[:, None] + shat_error * c[:, None] + \
        4 * U * (np.abs(g) + np.abs(shat) * c[:, None])
    dx = rms_backward(dy, gamma, shat, rstd, ds)[0]
    r, a = OUT_ROUND[dtype]
    e = e * rstd[:, None] + 2 * U * np.abs(dx)
    e = e + r * (np.abs(dx) + e) + a
    eg = (column_depth(N) + 2) * U * np.abs(dy * shat).sum(0) + (np.abs(dy) * shat_error).sum(0)
    return e, eg


# ------------------------------------------------------------------ 4 bits ----
MAGNITUDES = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])


def fp4_nearest(m):
    """Codes (0 to 7) of magnitudes: the nearest, of two as near the even one."""
    m = np.asarray(m, np.float64)
    off = np.abs(m[..., None] - MAGNITUDES)
    best = off.argmin(-1)                               # the lower of two as near
    other = np.minimum(best + 1, 7)
    tie = np.take_along_axis(off, other[..., None], -1)[..., 0] == off.min(-1)
    return np.where(tie & (best % 2 == 1), other, best)


def fp4_pack(x):
    """(codes 0..15 with the sign in bit 3, exps) of fp32-representable rows."""
    x = np.asarray(x, np.float64)
    N, K = x.shape
    G = -(-K // GROUP)
    code, exps = np.zeros((N, K), np.uint8), np.zeros((N, G), np.uint8)
    for g in range(G):
        v = x[:, g * GROUP:(g + 1) * GROUP]
        fine = np.isfinite(v).all(1)
        top = np.where(fine, np.abs(np.where(np.isfinite(v), v, 0)).max(1), 0)
        e = np.full(N, -126)
        while (up := top / 2.0 ** e >= 7.0).any():       # 7 lies between 6 and 8: to the even, 8
            e = e + up
        exps[:, g] = np.where(fine, e + 127, 255)
        c = fp4_nearest(np.abs(np.where(np.isfinite(v), v, 0)) / (2.0 ** e)[:, None])
        c = np.minimum(c, 7) | (np.signbit(v).astype(np.int64) << 3)
        code[:, g * GROUP:(g + 1) * GROUP] = np.where(fine[:, None], c, 0)
    return code, exps


def fp4_values(code, exps):
    step = np.where(exps == 255, np.nan, 2.0 ** (exps.astype(np.float64) - 127))
    sign = np.where(code >= 8, -1.0, 1.0)
    return sign * MAGNITUDES[code & 7] * np.repeat(step, GROUP, axis=1)[:, :code.shape[1]]


def fp4_codes(q, K):
    """The codes of packed bytes."""
    return np.stack((q & 15, q >> 4), 2).reshape(q.shape[0], -1)[:, :K]


def fp4_gemm(a, b, bias):
    return a @ b.T + bias


def fp4_gemm_bounds(a, b, bias, dtype):
    """Products are exact. The tensor core adds 64 of them at a time (a tree of six levels) to its
    sum, K / 64 times, and may truncate: 2 u an addition. The bias's addition rounds once."""
    s = np.abs(a) @ np.abs(b).T
    z = fp4_gemm(a, b, bias)
    e = 2 * (-(-a.shape[1] // 64) + 8) * U * s + U * np.abs(z)
    r, tiny = OUT_ROUND[dtype]
    return e + r * (np.abs(z) + e) + tiny


# -------------------------------------------------------- norm of many tensors ----
# A sum of at most 32 squares in two halves: a term passes 16 multiply-adds and one addition, so
# the sum of squares is within 17 u, its root within 8.5 u, and the norm rounds once more.
NORM_ERROR = 9.6 * U


def clip(tensors, max_norm):
    norm = np.sqrt(sum((t.astype(np.float64) ** 2).sum() for t in tensors))
    factor = max_norm / norm if norm > max_norm else 1.0
    return norm, [t.astype(np.float64) * factor for t in tensors]


def clip_bound(out, dtype):
    """The norm's error, the factor's rounding and the product's; then the type's."""
    r, a = OUT_ROUND[dtype]
    e = np.abs(out) * (8.6 * U + 2 * U)
    return e + r * (np.abs(out) + e) + a
