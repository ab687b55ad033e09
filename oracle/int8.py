"""CPU oracle for the 8-bit matrix product with scales and the quantisation of its rows -- TEST INFRASTRUCTURE, numpy only.

    S = sum_k A_ik W_jk                                   whole numbers, 64 bits
    y = fl(fl(fl(fl(S) sa_i) sw_j) + b_j)                 binary32, one rounding a step
    tau = Gamma(d)|v| [+ u (|v + b| + Gamma(d)|v|)]       extended precision, v = S sa sw, d = 2 (3 where |S| > 1/u)

The formula's value in extended precision carries errors of a few 2^-63, which the caller's comparison has to leave room for; it is
not rounded to binary32.
"""
import numpy as np


def _gamma(k, u, mode=0, lam=4.0):
    u = np.longdouble(u)
    if mode == 0:
        return k * u / (1 - k * u)
    return np.expm1(lam * np.sqrt(np.longdouble(k)) * u + k * u * u / (1 - u))


def quantize_rows(x):
    """(q, scale) of x [rows, cols], binary32 steps."""
    x = np.asarray(x, dtype=np.float32)
    m = np.abs(x).max(axis=1, initial=0) if x.shape[1] else np.zeros(x.shape[0], np.float32)
    finite = np.isfinite(x).all(axis=1)
    scale = np.where(finite, np.where(finite, m, 0).astype(np.float32) * (np.float32(1) / np.float32(127)), np.float32(np.nan)).astype(np.float32)
    some = scale > 0                                         # (NaN compares false)
    with np.errstate(invalid="ignore", over="ignore"):
        q = np.clip(np.rint(np.where(some[:, None], x, 0) / np.where(some, scale, 1)[:, None].astype(np.float32)), -127, 127)
    return q.astype(np.int8), scale


def linear_int8(A, sa, W, sw, bias=None, model=None):
    """(y, tau): y binary32, tau extended precision; A [M, K], W [N, K]."""
    u, mode, lam, flags = (2.0 ** -24, 0, 4.0, 0) if model is None else (model.u, model.mode, model.lam, model.flags)
    S = A.astype(np.int64) @ W.astype(np.int64).T
    sa, sw = np.asarray(sa, np.float32)[:, None], np.asarray(sw, np.float32)[None, :]
    with np.errstate(all="ignore"):
        y = (S.astype(np.float32) * sa) * sw
        if bias is not None:
            y = y + np.asarray(bias, np.float32)[None, :]
        L = np.longdouble
        v = S.astype(L) * sa.astype(L) * sw.astype(L)
        g = np.where(np.abs(S).astype(L) * L(u) > 1, _gamma(3, u, mode, lam), _gamma(2, u, mode, lam))
        tau = g * np.abs(v)
        if bias is not None:
            tau = tau + L(u) * (np.abs(v + np.asarray(bias, np.float32).astype(L)[None, :]) + tau)
        if flags & 1:
            tau = tau + (np.abs(S) + np.abs(sa).astype(L) + np.abs(sw).astype(L) + 1) * L(2) ** -149
        finite = np.isfinite(sa) & np.isfinite(sw)
        if bias is not None:
            finite = finite & np.isfinite(np.asarray(bias, np.float32))[None, :]
        tau = np.where(finite, tau, L(np.nan))               # (finite operands beyond the binary32 range keep their value)
    assert y.dtype == np.float32
    return y, tau
