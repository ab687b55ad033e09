"""The oracles of the rotary tables, the norm and rotation of heads and the product with 4-bit weights: closed forms, the existing oracles where
they meet, and executions in binary32 of every kind that the bounds say they cover."""
import numpy as np
import pytest

import oracle
from oracle import int4, rotary

F, L, U = np.float32, np.longdouble, 2.0 ** -24


def test_reduction_of_far_angles():
    # cos(n) for whole angles, from the published value of cos(10^22)-like hard cases inside the range, and the addition theorem
    c, s, _, _ = rotary.rope_tables([0, 1, 2, 3, 10 ** 6, 10 ** 6 + 1, -7, 2 ** 40], np.array([1.0], F))
    assert c[0, 0] == 1 and s[0, 0] == 0
    assert abs(c[1, 0] - L("0.54030230586813971740093660744297660373")) < 1e-18
    assert abs(s[1, 0] - L("0.84147098480789650665250232163029899962")) < 1e-18
    assert abs(c[5, 0] - (c[4, 0] * c[1, 0] - s[4, 0] * s[1, 0])) < 1e-17
    assert abs(c[6, 0] - np.cos(L(7))) < 1e-17 and abs(s[6, 0] + np.sin(L(7))) < 1e-17
    assert np.abs(c * c + s * s - 1).max() < 1e-17


def test_small_negative_angles():
    """The sine is odd, and next to 0 it is the angle, to all bits of an angle of any size and sign."""
    f = np.array([1e-45, 1e-40, 1e-30, 2.0 ** -70, 1e-19, 3e-10, 0.25], F)
    c, s, tc, ts = rotary.rope_tables([7, 70001], f)
    c2, s2, tc2, ts2 = rotary.rope_tables([-7, -70001], f)
    for a, b in ((c, c2), (s, -s2), (tc, tc2), (ts, ts2)):
        assert np.array_equal(a, b)
    angle = -np.array([[7], [70001]]).astype(L) * f[None, :5].astype(L)
    assert (np.abs(s2[:, :5] / angle - 1) < 2.0 ** -60).all()
    # angles a little below a multiple of 2 pi
    near = np.nextafter((2 * np.pi * np.arange(1, 50)).astype(F), F(0))
    s3 = rotary.rope_tables([1], near)[1]
    assert (np.abs(s3 - np.sin(near.astype(L))) < 2.0 ** -58).all() and np.array_equal(s3, -rotary.rope_tables([-1], near)[1])


@pytest.mark.parametrize("scale", [1.0, 1.25, -0.7])
def test_tables_cover_executions(scale):
    rng = np.random.default_rng(3)
    p = np.concatenate([np.arange(40), rng.integers(0, 200000, 200), [2 ** 24 + 1, 2 ** 25 + 3]])
    f = (1e6 ** -np.linspace(0, 1, 32)).astype(F)
    c, s, tc, ts = rotary.rope_tables(p, f, scale)
    angle32 = p.astype(F)[:, None] * f[None, :]              # a rounding for p beyond 2^24, one for the product
    angle64 = p.astype(np.float64)[:, None] * f.astype(np.float64)[None, :]
    for angle in (angle32.astype(np.float64), angle64):
        for v, t, fn in ((c, tc, np.cos), (s, ts, np.sin)):
            y = fn(angle).astype(F) if scale == 1.0 else F(scale) * fn(angle).astype(F)
            assert (np.abs(y.astype(L) - v) <= t).all()
    # far angles of positions that are not rounded: little beside the angle's one rounding and the function's own error is left in the bound
    far = (np.abs(angle64) > 1000) & (p <= 2 ** 24)[:, None]
    assert (tc[far] <= 1.01 * abs(scale) * (1.01 * U * np.abs(angle64[far]) + 5 * U + (0 if scale == 1 else 1.1 * U))).all()


def test_heads_without_norm_are_the_rotary_oracle():
    rng = np.random.default_rng(0)
    x = rng.normal(0, 1, (5, 3, 16)).astype(F)
    c, s = rng.uniform(-1, 1, (2, 7, 8)).astype(F)
    for inter in (False, True):
        _, tau = rotary.norm_rope(x, c, s, 16, norm=False, interleaved=inter)
        old = oracle.bound_rope(x.reshape(15, 16), c, s, inner=3, interleaved=inter)
        new = tau.reshape(15, 16)
        # (the C oracle rounds up to binary32; g2 there includes the same Gamma(2))
        assert (old.astype(L) >= new * (1 - 1e-15)).all() and (old.astype(L) <= new * (1 + 1.3e-7)).all()


def test_heads_without_rotation_are_the_rmsnorm_oracle():
    rng = np.random.default_rng(1)
    x, g = rng.normal(0, 2, (4, 3, 24)).astype(F), rng.normal(1, 0.2, 24).astype(F)
    none = np.empty((1, 0), F)
    _, tau = rotary.norm_rope(x, none, none, 0, gamma_q=g, eps=1e-6)
    old = oracle.bound_norm(oracle.RMSNORM, x.reshape(12, 24), y=None, g=g, eps=1e-6).astype(L)
    assert (old >= tau.reshape(12, 24) * (1 - 1e-15)).all() and (old <= tau.reshape(12, 24) * (1 + 1.5e-7)).all()


@pytest.mark.parametrize("d,rot,inter,norm", [(8, 8, False, True), (16, 4, True, True), (128, 128, False, True), (64, 32, False, False), (2, 2, True, True)])
def test_heads_cover_executions(d, rot, inter, norm):
    rng = np.random.default_rng(d + rot)
    T, H, npos = 60, 4, 9
    x = (rng.normal(0, 1, (T, H, d)) * np.exp(rng.normal(0, 1, (T, H, 1)))).astype(F)
    g = rng.normal(1, 0.3, d).astype(F) if norm else None
    cd, sd, tc, ts = rotary.rope_tables(rng.integers(0, 5000, npos), (1e4 ** -np.linspace(0, 1, rot // 2)).astype(F))
    # tables of another execution than the verifier's, inside their bounds
    c, s = cd.astype(F), sd.astype(F)
    c2 = (cd + 0.9 * tc * rng.choice([-1, 1], tc.shape)).astype(F)
    s2 = (sd + 0.9 * ts * rng.choice([-1, 1], ts.shape)).astype(F)
    tcu, tsu = (np.nextafter((t + np.abs(a.astype(L) - b)).astype(F), F(1)) for t, a, b in ((tc, c, cd), (ts, s, sd)))
    y, tau = rotary.norm_rope(x, c, s, rot, gamma_q=g, norm=norm, tau_cos=tcu, tau_sin=tsu, interleaved=inter)
    at = np.arange(T) % npos
    ia, ib = (np.arange(0, rot, 2), np.arange(1, rot, 2)) if inter else (np.arange(rot // 2), np.arange(rot // 2) + rot // 2)
    for order in range(4):
        h = x
        if norm:
            sq = x * x
            perm = rng.permutation(d)
            v = np.add.accumulate(sq[..., perm], axis=-1, dtype=F)[..., -1:] if order % 2 else sq.sum(-1, keepdims=True, dtype=F)
            v = v * F(1 / d) if order < 2 else v / F(d)
            r = F(1) / np.sqrt(v + F(1e-6))
            h = g * (x * r) if order < 2 else (x * r) * g
        for cc, ss in ((c, s), (c2, s2)):
            out = h.copy()
            C, S = cc[at][:, None, :], ss[at][:, None, :]
            fused = lambda a, b, e, f_: (a.astype(L) * b + (e * f_).astype(L)).astype(F)
            if order % 2:
                out[..., ia], out[..., ib] = fused(h[..., ia], C, -h[..., ib], S), fused(h[..., ib], C, h[..., ia], S)
            else:
                out[..., ia], out[..., ib] = h[..., ia] * C - h[..., ib] * S, h[..., ib] * C + h[..., ia] * S
            assert (np.abs(out.astype(L) - y) <= tau).all()


def test_int4_against_the_matmul_oracle():
    rng = np.random.default_rng(2)
    A, q, s = rng.normal(0, 1, (3, 50)).astype(F), rng.integers(0, 16, (7, 50)), np.full((7, 2), 2.0 ** -5, F)
    y, tau, size = int4.linear_int4(A, q, s, 32)
    W = ((q - 8) * 2.0 ** -5).astype(F)                      # exact, so the bounds differ by the one rounding that the scale may cost
    old = oracle.bound_linear(A, W).astype(L)
    assert (np.abs(tau / old * (50 * (1 - 51 * U)) / (51 * (1 - 50 * U)) - 1) < 1.3e-7).all()
    assert np.abs(y - A.astype(L) @ W.astype(L).T).max() < 1e-15


@pytest.mark.parametrize("K,group", [(1, 32), (2, 2), (33, 32), (64, 32), (300, 64), (257, 257)])
@pytest.mark.parametrize("with_bias", [False, True])
def test_int4_covers_executions(K, group, with_bias):
    rng = np.random.default_rng(K)
    M, N, G = 5, 9, -(-K // group)
    A = (rng.normal(0, 1, (M, K)) * np.exp(rng.normal(0, 2, (M, K)))).astype(F)
    q, z = rng.integers(0, 16, (N, K)), rng.integers(0, 16, (N, G)).astype(np.uint8)
    s = rng.uniform(0.001, 0.1, (N, G)).astype(F)
    b = rng.normal(0, 0.1, N).astype(F) if with_bias else None
    y, tau, _ = int4.linear_int4(A, q, s, group, z, b)
    of = np.arange(K) // group
    d = (q - z.astype(int)[:, of]).astype(F)
    w = d * s[:, of]
    runs = []
    for perm in (np.arange(K), rng.permutation(K), np.argsort(-np.abs(A[0]))):
        t = F(0) * np.zeros((M, N), F)
        for k in perm:                                       # weights first, one sum
            t = t + A[:, k, None] * w[None, :, k]
        runs.append(t if b is None else t + b)
        t = np.zeros((M, N), F) if b is None else np.broadcast_to(b, (M, N)).astype(F)
        for g in range(G):                                   # a group's sum, then its scale, the bias first
            part = np.zeros((M, N), F)
            for k in range(g * group, min(K, (g + 1) * group)):
                part = part + A[:, k, None] * d[None, :, k]
            t = t + part * s[None, :, g]
        runs.append(t)
    for t in runs:
        assert t.dtype == F and (np.abs(t.astype(L) - y) <= tau).all()


def test_packing():
    q = np.array([[1, 2, 3], [15, 0, 7]])
    assert int4.pack(q).tolist() == [[0x21, 0xF3], [0x0F, 0xF7]]
