"""The oracles of the 8-bit product, the row quantisation and the channels-last GroupNorm with an activation, pinned without a GPU: every
execution the operator admits lies within the bound, closed forms, and agreement with the layouts the C oracle knows."""
import itertools
from fractions import Fraction

import numpy as np
import pytest

import oracle
from oracle import groupnorm_act as gn
from oracle import int8

U = 2.0 ** -24


def _round(q):
    """A rational rounded to binary32, to nearest, ties to even (normal range)."""
    f = np.float32(float(q))                                 # within one step of q; the nearest is among its neighbours
    near = [np.nextafter(f, np.float32(-np.inf)), f, np.nextafter(f, np.float32(np.inf))]
    return Fraction(float(min(near, key=lambda v: (abs(Fraction(float(v)) - q), int(v.view(np.uint32)) & 1))))


def _executions(S, sa, sw, b):
    """Both orders of the scales, and their product first; with and without a fused last step."""
    s, sa, sw = Fraction(int(S)), Fraction(float(sa)), Fraction(float(sw))
    f = _round(s)
    for first, second in ((sa, sw), (sw, sa)):
        part = _round(f * first)
        yield from ([_round(part * second)] if b is None else [_round(_round(part * second) + b), _round(part * second + b)])
    scale = _round(sa * sw)
    yield from ([_round(f * scale)] if b is None else [_round(_round(f * scale) + b), _round(f * scale + b)])


@pytest.mark.parametrize("K,with_bias", [(1, False), (7, True), (64, True), (1100, False), (20000, True)])
def test_every_execution_of_the_8_bit_product_is_within_its_bound(K, with_bias):
    rng = np.random.default_rng(K)
    A, W = rng.integers(-128, 128, (6, K), dtype=np.int8), rng.integers(-128, 128, (9, K), dtype=np.int8)
    A[0], W[0] = -128, -128                                  # the largest sum there is
    sa, sw = rng.uniform(0.001, 0.1, 6).astype(np.float32), rng.uniform(-0.1, 0.1, 9).astype(np.float32)
    bias = rng.normal(0, 1, 9).astype(np.float32) if with_bias else None
    y, tau = int8.linear_int8(A, sa, W, sw, bias)
    S = A.astype(np.int64) @ W.astype(np.int64).T
    for i, j in itertools.product(range(6), range(9)):
        b = None if bias is None else Fraction(float(bias[j]))
        true = Fraction(int(S[i, j])) * Fraction(float(sa[i])) * Fraction(float(sw[j])) + (b or 0)
        runs = list(_executions(S[i, j], sa[i], sw[j], b))
        assert Fraction(float(y[i, j])) in runs              # the re-executed output is one of them
        assert all(abs(r - true) <= Fraction(float(tau[i, j])) * (1 + Fraction(1, 1 << 50)) for r in runs)
    if bias is None and K == 1:                              # closed form: two roundings
        assert float(tau[0, 0]) == pytest.approx(2 * U / (1 - 2 * U) * 16384 * float(sa[0]) * abs(float(sw[0])), rel=1e-15)


def test_quantised_rows_are_within_half_a_step_and_keep_their_largest_element():
    rng = np.random.default_rng(1)
    x = (rng.normal(0, 1, (40, 333)) * np.exp(rng.normal(0, 6, (40, 1)))).astype(np.float32)
    x[0] = 0; x[1, 5] = np.inf; x[2, 7] = np.nan; x[3] = 0; x[3, 3] = 1e-45; x[4] = 0; x[4, 0] = -3.0
    q, s = int8.quantize_rows(x)
    good = [r for r in range(40) if r not in (0, 1, 2, 3)]
    assert (q[[0, 1, 2, 3]] == 0).all() and s[0] == 0 and np.isnan(s[1]) and np.isnan(s[2]) and s[3] == 0
    assert (np.abs(q[good]).max(axis=1) == 127).all() and q[4, 0] == -127
    # |x/s - q| <= 1/2 and the quotient's own rounding, 127 2^-24 at most
    assert (np.abs(x[good].astype(np.longdouble) / s[good, None] - q[good]) <= 0.5 + 127 * U).all()


@pytest.mark.parametrize("act", [gn.NONE, gn.RELU, gn.SILU])
@pytest.mark.parametrize("P,C,groups", [(1, 4, 1), (5, 6, 3), (16, 8, 2), (3, 5, 5)])
def test_binary32_executions_of_the_group_norm_are_within_the_bound(act, P, C, groups):
    rng = np.random.default_rng(P * 100 + C)
    per, f = C // groups, np.float32
    for scale, shift in ((1.0, 0.0), (1e-3, 1.0), (30.0, -5.0)):
        x = (rng.normal(shift, scale, (2, P, C))).astype(f)
        gamma, beta = rng.normal(1, 0.3, C).astype(f), rng.normal(0, 0.5, C).astype(f)
        y, tau, _ = gn.groupnorm_act(act, x, groups, gamma, beta, 1e-5)
        for order in (1, -1):
            X = x.reshape(2, P, groups, per)
            n = f(P * per)

            def total(t):
                rows = np.ascontiguousarray(np.moveaxis(t, 2, 1)).reshape(2, groups, -1)[..., ::order]
                acc = np.zeros((2, groups), f)
                for i in range(rows.shape[-1]):
                    acc = acc + rows[..., i]
                return acc[:, None, :, None]
            mu = total(X) / n
            d = X - mu
            r = f(1) / np.sqrt(total(d * d) / n + f(1e-5))
            p = (d * r * gamma.reshape(1, 1, groups, per) + beta.reshape(1, 1, groups, per)).reshape(2, P, C)
            assert p.dtype == f
            if act == gn.SILU:
                run = p / (f(1) + np.exp(-p))
            elif act == gn.RELU:
                run = np.maximum(p, f(0))
            else:
                run = p
            assert (np.abs(run.astype(np.longdouble) - y) <= tau).all()


def test_slope_bounds_of_silu():
    t = np.linspace(-40, 40, 400001).astype(np.longdouble)
    sig = 1 / (1 + np.exp(-t))
    first = sig * (1 + t * (1 - sig))
    second = sig * (1 - sig) * (2 + t * (1 - 2 * sig))
    assert np.abs(first).max() < 1.1 and np.abs(second).max() <= 0.5
    assert np.abs(np.diff(first) / np.diff(t)).max() <= 0.5


def test_one_group_of_one_pixel_is_a_layernorm_row():
    rng = np.random.default_rng(9)
    x, gamma, beta = (rng.normal(0.3, 1, s).astype(np.float32) for s in ((7, 1, 48), (48,), (48,)))
    y, tau, _ = gn.groupnorm_act(gn.NONE, x, 1, gamma, beta, 1e-5)
    row = oracle.bound_norm(oracle.LAYERNORM, x.reshape(7, 48), y=y.reshape(7, 48).astype(np.float32), g=gamma, b=beta, eps=1e-5)
    # the C oracle's last rounding is u|y| of the computed output, this one's u(|p| + E_p): apart by u E_p and u (half a step of y)
    assert np.allclose(row, tau.reshape(7, 48).astype(np.float64), rtol=4e-7, atol=0)


def test_constant_groups_have_a_bound_from_eps_and_rows_without_eps_have_none():
    x = np.full((1, 4, 6), 2.0, np.float32)
    y, tau, _ = gn.groupnorm_act(gn.NONE, x, 2, None, None, 1e-2)
    assert (y == 0).all() and np.isfinite(tau.astype(np.float64)).all() and (tau > 0).all()
    assert np.isnan(gn.groupnorm_act(gn.NONE, x, 2, None, None, 0.0)[1].astype(np.float64)).all()
