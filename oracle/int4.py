"""CPU oracle for the product with 4-bit weights and group scales -- TEST INFRASTRUCTURE, numpy only, in extended precision.

    w = (q - z) s,  y = sum a w + b,  tau = Gamma(K')(sum |a||w| + |b|),  K' = K + 1 (K + 2 with a bias)
"""
import numpy as np

from .int8 import _gamma

L = np.longdouble


def pack(q):
    """Whole numbers 0 .. 15 [N, K] as bytes [N, (K + 1) / 2], the even column in the low four bits (a column of 15 behind an odd K)."""
    q = np.asarray(q, np.uint8)
    if q.shape[1] % 2:
        q = np.concatenate([q, np.full((len(q), 1), 15, np.uint8)], axis=1)
    return np.ascontiguousarray(q[:, 0::2] | q[:, 1::2] << 4)


def linear_int4(A, q, scale, group, zero=None, bias=None, model=None):
    """(y, tau, size): the formulas' values and sum |a||w| + |b|; A [M, K], q [N, K] whole numbers, scale and zero [N, G]."""
    u, mode, lam, flags = (2.0 ** -24, 0, 4.0, 0) if model is None else (model.u, model.mode, model.lam, model.flags)
    M, K = A.shape
    of = np.arange(K) // group
    with np.errstate(all="ignore"):
        z = np.full(scale.shape, 8) if zero is None else zero.astype(np.int64)
        w = (q.astype(np.int64) - z[:, of]).astype(L) * scale.astype(L)[:, of]
        a = A.astype(L)
        y, size = a @ w.T, np.abs(a) @ np.abs(w).T
        steps = K + 1
        if bias is not None:
            y, size, steps = y + bias.astype(L)[None, :], size + np.abs(bias.astype(L))[None, :], steps + 1
        tau = _gamma(steps, u, mode, lam) * size
        if flags & 1:
            tau = tau + L(2) ** -149 * (steps + np.abs(a).sum(1)[:, None] + np.abs(scale.astype(L))[:, of].sum(1)[None, :])
        tau = np.where(np.isfinite(size), tau, L(np.nan))    # (finite operands stay inside the extended range)
    return y, tau, size
