"""CPU oracle for the rotary tables and for the norm and rotation of query and key heads -- TEST INFRASTRUCTURE, numpy only: the formulas
step by step, in extended precision (errors of a few n 2^-64, which the caller's comparison leaves room for; not rounded to binary32).

    tables    c = m cos(p f); E = Gamma(d)|p f|; B = min(|sin| E + E^2/2, E, 1 + |cos|); B' = B + c_cos u(|cos| + B); tau = |m| (B' [+ u(|cos| + B')])
    heads     E_t, E_v, E_w, w_lo, E_r, R of the RMSNORM chain; E = |x g|(E_r + u R) + u |x g| R (1+u)^2; then every pair's two products
"""
import numpy as np

from .int8 import _gamma

L = np.longdouble
# 2 pi with 128 bits, as three parts whose products with whole numbers below 2^40 are exact in extended precision
_TWO_PI = int("6487ed5110b4611a62633145c06e0e68948127044533e63a0105df531d89cd91", 16)      # floor(2 pi 2^252)


def _reduced(p, f):
    """p f - 2 pi n for whole p and binary32 f, from exact whole-number arithmetic; one element at a time."""
    if not np.isfinite(f):
        return L(np.nan)
    num, den = float(f).as_integer_ratio()
    num *= int(p)
    t = (abs(num) << 252) // den                             # (of magnitudes: below 0 the two parts at the end would take from each other, and a small angle's bits with them)
    r = t % _TWO_PI
    sign = 1 if num >= 0 else -1
    if r > _TWO_PI // 2:
        r, sign = _TWO_PI - r, -sign
    hi = r >> 190                                            # 64 bits at a time
    return sign * (L(hi) * L(2) ** -62 + L(r - (hi << 190)) * L(2) ** -252)


def rope_tables(positions, inv_freq, scale=1.0, model=None):
    """(cos, sin, tau_cos, tau_sin), [npos, half]."""
    u, mode, lam = (2.0 ** -24, 0, 4.0) if model is None else (model.u, model.mode, model.lam)
    c_cos, c_sin = (4.0, 4.0) if model is None else (model.c_cos, model.c_sin)
    p, f, m = np.asarray(positions, np.int64), np.asarray(inv_freq, np.float32), L(np.float32(scale))
    theta = np.array([[_reduced(a, b) for b in f] for a in p], dtype=L).reshape(len(p), len(f))
    angle = np.abs(p.astype(L)[:, None] * f.astype(L)[None, :])
    u = L(u)
    E = np.where(np.abs(p.astype(L))[:, None] * u > 1, _gamma(2, u, mode, lam), _gamma(1, u, mode, lam)) * angle
    c, s = np.cos(theta), np.sin(theta)
    out = []
    for v, slope, lib in ((c, s, L(c_cos)), (s, c, L(c_sin))):
        B = np.minimum(np.minimum(np.abs(slope) * E + E * E / 2, E), 1 + np.abs(v))
        B = B + lib * u * (np.abs(v) + B)
        out.append(np.abs(m) * (B if m == 1 else B + u * (np.abs(v) + B)))
    return m * c, m * s, out[0], out[1]


def norm_rope(x, cos, sin, rot, gamma_q=None, gamma_k=None, heads_k=0, eps=1e-6, norm=True, tau_cos=None, tau_sin=None, positions=None,
              interleaved=False, model=None):
    """(y, tau) of x [tokens, heads, d]."""
    u, mode, lam, flags = (2.0 ** -24, 0, 4.0, 0) if model is None else (model.u, model.mode, model.lam, model.flags)
    c_div, c_rsqrt = (2.0, 2.0) if model is None else (model.c_div, model.c_rsqrt)
    u, cd, cr = L(u), L(c_div), L(c_rsqrt)
    T, H, d = x.shape
    npos = len(cos)
    at = np.arange(T) % npos if positions is None else np.asarray(positions)
    inside = (at >= 0) & (at < npos)
    at = np.where(inside, at, 0)
    with np.errstate(all="ignore"):
        X = x.astype(L)
        g = np.ones((H, d), L)
        if gamma_q is not None:
            g[:H - heads_k] = gamma_q.astype(L)
        if gamma_k is not None:
            g[H - heads_k:] = gamma_k.astype(L)
        if norm:
            G = _gamma(d - 1, u, mode, lam)
            S = (X * X).sum(-1, keepdims=True)
            E_t = (G * (1 + u) + u) * S
            v = S / d
            E_v = (E_t / d + cd * u * v) / (1 - cd * u)
            w = v + L(np.float32(eps))
            E_w = (E_v + u * w) / (1 - u)
            w_lo = np.where(w > E_w, w - E_w, L(np.nan))
            r = 1 / np.sqrt(w)
            E_r = E_w / (2 * w_lo * np.sqrt(w_lo)) + cr * u / np.sqrt(w_lo)
            R = r + E_r
            h = X * g * r
            E = np.abs(X * g) * (E_r + u * R) + u * np.abs(X * g) * R * (1 + u) ** 2
        else:
            h, E = X, X * 0                                  # (NaN where x is not finite)
        y, tau = h.copy(), E.copy()
        if rot:
            ia, ib = (np.arange(0, rot, 2), np.arange(1, rot, 2)) if interleaved else (np.arange(rot // 2), np.arange(rot // 2) + rot // 2)
            c, s = (np.where(inside[:, None], t[at].astype(L), L(np.nan))[:, None, :] for t in (cos, sin))
            tc, ts = (L(0), L(0)) if tau_cos is None else (np.abs(t[at].astype(L))[:, None, :] for t in (tau_cos, tau_sin))
            g2 = _gamma(2, u, mode, lam)
            ha, hb, Ea, Eb = h[..., ia], h[..., ib], E[..., ia], E[..., ib]
            big = lambda v, e, t, et: (np.abs(v) + e) * (np.abs(t) + et)
            off = lambda v, e, t, et: e * (np.abs(t) + et) + np.abs(v) * et
            low = L(2) ** -148 if flags & 1 else L(0)
            y[..., ia], y[..., ib] = ha * c - hb * s, hb * c + ha * s
            tau[..., ia] = off(ha, Ea, c, tc) + off(hb, Eb, s, ts) + g2 * (big(ha, Ea, c, tc) + big(hb, Eb, s, ts)) + low
            tau[..., ib] = off(hb, Eb, c, tc) + off(ha, Ea, s, ts) + g2 * (big(hb, Eb, c, tc) + big(ha, Ea, s, ts)) + low
        tau = np.where(np.isfinite(tau), tau, L(np.nan))
    return y, tau
