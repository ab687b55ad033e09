"""CPU oracle for GroupNorm with an activation on channels-last features -- TEST INFRASTRUCTURE, numpy only: the chain of the two-pass
algorithm step by step (the steps and names of oracle/tao_oracle.c's LAYERNORM), in extended precision, element by element.

The formulas' values in extended precision carry errors of a few n 2^-64; they are not rounded to binary32.
"""
import numpy as np

from .int8 import _gamma

NONE, RELU, SILU = "none", "relu", "silu"


def groupnorm_act(act, x, groups, gamma=None, beta=None, eps=1e-5, model=None):
    """(y, tau, E) of x [batch, positions, channels]: exact output, bound, and the bound of the activation's argument."""
    L = np.longdouble
    u, mode, lam = (2.0 ** -24, 0, 4.0) if model is None else (model.u, model.mode, model.lam)
    c_div, c_rsqrt, c_exp = (2.0, 2.0, 2.0) if model is None else (model.c_div, model.c_rsqrt, model.c_exp)
    u, cd, cr, ce = L(u), L(c_div), L(c_rsqrt), L(c_exp)
    B, P, C = x.shape
    per = C // groups
    n = P * per
    G = _gamma(n - 1, u, mode, lam)
    eps = L(np.float32(eps))
    with np.errstate(all="ignore"):
        X = x.astype(L).reshape(B, P, groups, per)
        over = lambda t: t.sum(axis=(1, 3), keepdims=True)
        mu = over(X) / n
        E_mu = (G * over(np.abs(X)) / n + cd * u * np.abs(mu)) / (1 - cd * u)
        d = X - mu
        ad = np.abs(d)
        E_d = (E_mu + u * ad) / (1 - u)
        D = ad + E_d
        E_t = G * over(D * D * (1 + u)) + over(E_d * (ad + D) + u * D * D)
        v = over(d * d) / n
        E_v = (E_t / n + cd * u * v) / (1 - cd * u)
        w = v + eps
        E_w = (E_v + u * w) / (1 - u)
        w_lo = np.where(w > E_w, w - E_w, L(np.nan))
        r = 1 / np.sqrt(w)
        E_r = E_w / (2 * w_lo * np.sqrt(w_lo)) + cr * u / np.sqrt(w_lo)
        R = r + E_r
        E_h = D * E_r + r * E_d + u * D * R
        g = L(1) if gamma is None else gamma.astype(L).reshape(1, 1, groups, per)
        b = L(0) if beta is None else beta.astype(L).reshape(1, 1, groups, per)
        E_p = np.abs(g) * E_h + u * np.abs(g) * (ad * r + E_h)
        p = d * r * g + b
        E = np.where(np.isfinite(g) & np.isfinite(b), E_p + u * (np.abs(p) + E_p), L(np.nan))
        if act == SILU:
            sig = 1 / (1 + np.exp(-p))
            y = p * sig
            slope = np.abs(sig * (1 + p / (1 + np.exp(p))))
            Bd = np.minimum(slope * E + E * E / 4, L(11) / 10 * E)
            omega = (ce * u / (1 - ce * u) + u) / (1 - u)
            f = omega / (1 - u) + u
            tau = Bd + f / (1 - f) * (np.abs(y) + Bd)
        elif act == RELU:
            y = np.maximum(p, 0)
            tau = np.maximum(np.minimum(E, p + E), 0)
        else:
            y, tau = p, E
    flat = lambda t: np.broadcast_to(t, X.shape).reshape(B, P, C)
    return flat(y), flat(tau), flat(E)
