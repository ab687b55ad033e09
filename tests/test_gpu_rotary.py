"""Rotary tables, and the norm and rotation of query and key heads, against their oracles: outputs within one rounding of the formula, bounds
one-sided within 1e-6, profiles equal to the streaming check of the stored output and bound."""
import numpy as np
import pytest
import torch

import oracle
from oracle import rotary
from opmap import assert_profile_equal
from test_gpu_int8 import assert_bound, cuda

pytestmark = pytest.mark.gpu
F, L, U = np.float32, np.longdouble, 2.0 ** -24


@pytest.fixture(scope="module")
def tao():
    import paper_2510_16028_amd as t
    return t


def assert_rounded(y, exact, slack, what=""):
    """The formula's value rounded once: half a step of binary32 (2^-150 where it is subnormal), and what binary64 leaves open (slack)."""
    y, e = y.astype(L), np.asarray(exact)
    assert np.array_equal(np.isnan(y), np.isnan(e)), what
    # (from (2 - 2^-24) 2^127 on, half a step above the largest binary32 value, rounding to nearest gives infinity: next to it either is right)
    edge = (2 - L(2) ** -24) * L(2) ** 127
    beyond = np.abs(e) > edge * (1 + L(2) ** -40)
    assert np.isinf(y[beyond]).all(), what
    ok = np.abs(e) < edge * (1 - L(2) ** -40)
    slack = np.broadcast_to(slack, e.shape)[ok]
    assert (np.abs(y[ok] - e[ok]) <= np.abs(e[ok]) * L(U) * (1 + L(2) ** -20) + slack + L(2) ** -149).all(), what


# ------------------------------------------------------------------ tables

def frequencies(half, theta=1e6):
    return (theta ** (-np.arange(half) / max(half, 1))).astype(F)


def assert_tables(got, p, f, scale=1.0, model=None):
    exact = rotary.rope_tables(p, f, scale, model)
    far = np.abs(p.astype(L)[:, None] * f.astype(L)[None, :])
    for g, e in zip(got[:2], exact[:2]):
        assert_rounded(g.cpu().numpy(), e, abs(L(F(scale))) * (L(2) ** -44 + far * L(2) ** -52))
    for g, e in zip(got[2:], exact[2:]):
        assert_bound(g.cpu().numpy(), e)


@pytest.mark.parametrize("npos,half", [(1, 1), (1, 64), (3, 5), (64, 64), (100, 33), (257, 16), (5, 300)])
@pytest.mark.parametrize("scale", [1.0, 1.3465735902799727, -0.5, 0.0])
def test_tables(tao, npos, half, scale):
    rng = np.random.default_rng(npos + half)
    p, f = rng.integers(0, 200000, npos), frequencies(half)
    assert_tables(tao.tao_bound_rope_tables(*cuda(f, p), scale=scale), p, f, scale)


def test_tables_of_positions_in_order(tao):
    f = frequencies(24)
    got = tao.tao_bound_rope_tables(cuda(f)[0], npos=211)
    assert_tables(got, np.arange(211), f)
    given = tao.tao_bound_rope_tables(cuda(f)[0], torch.arange(211, device="cuda"))
    for a, b in zip(got, given):
        assert torch.equal(a, b)
    assert bool((got[0][0] == 1).all()) and bool((got[1][0] == 0).all()) and bool((got[3][0] == 0).all())      # the sine of 0 is exact


def test_tables_of_far_negative_and_rounded_positions(tao):
    p = np.array([0, -1, -7, 2 ** 24 - 1, 2 ** 24, 2 ** 24 + 1, -2 ** 24 - 1, 2 ** 31, 2 ** 40, -2 ** 45])
    f = np.array([1.0, 0.1, 3e-7, 1e-12, 1e-30, 1e-45, 0.0, -0.25, 31.0], F)
    assert_tables(tao.tao_bound_rope_tables(*cuda(f, p)), p, f)


def test_tables_next_to_the_zeros(tao):
    """Angles next to multiples of pi/2: the smaller of the two functions is what the reduction leaves."""
    k = np.arange(1, 400)
    f = np.concatenate([(k * np.pi / 2).astype(F), np.nextafter((k * np.pi / 2).astype(F), F(0)), (np.pi / 4 * (2 * k + 1)).astype(F)])
    p = np.array([1, 3])
    assert_tables(tao.tao_bound_rope_tables(*cuda(f, p)), p, f)


def test_tables_of_angles_whose_products_round(tao):
    """Odd far positions and frequencies of 24 bits, so that p f has more than 53: what the product leaves off is part of every table and bound; positions that binary64 does not hold, up to the ends of int64."""
    rng = np.random.default_rng(7)
    f = np.array([1.0, 0.1, 1 / 3, 0.731, 0.999, -0.25], F)
    for bits in (20, 24, 28, 29, 30, 32, 34, 36, 40, 44, 45, 48, 49):
        p = np.concatenate([rng.integers(2 ** (bits - 1), 2 ** bits, 24) | 1, [2 ** bits + 1, 2 ** bits - 3, -2 ** bits + 1]])
        assert_tables_closely(tao, p, f)
    k = np.arange(1, 200)
    near = np.concatenate([(k * np.pi / 2).astype(F), (k * np.pi / 4).astype(F)])         # one of the two functions is next to 0 at p = 1, 3, 5
    assert_tables_closely(tao, np.array([1, 3, 5, 999999999, 2 ** 36 + 1, 2 ** 40 - 3]), near)
    for bits in (54, 58, 63):
        p = rng.integers(2 ** (bits - 1), 2 ** bits - 1, 20) | 1
        p = np.concatenate([p, -p])
        assert_tables_closely(tao, p, (f[1:] * 2.0 ** (48 - bits)).astype(F))
        assert_tables_closely(tao, p, (f[1:] * 2.0 ** (20 - bits)).astype(F))
    ends = np.array([2 ** 63 - 1, 2 ** 63 - 512, 2 ** 63 - 513, 2 ** 63 - 1025, -2 ** 63, -2 ** 63 + 1, 2 ** 53, 2 ** 53 + 1, -2 ** 53 - 1])
    assert_tables_closely(tao, ends, np.array([2.0 ** -14, 0.7 * 2.0 ** -14, 1e-10, 1e-19], F))


def assert_tables_closely(tao, p, f, scale=1.0, model=None):
    """As the header has it: the formula to |m| 2^-44, from angles of 2^45 on to |m| 2^-34, rounded once; bounds as everywhere."""
    got, exact = tao.tao_bound_rope_tables(*cuda(f, p), scale=scale, model=model), rotary.rope_tables(p, f, scale, model)
    far = np.abs(p.astype(L)[:, None] * f.astype(L)[None, :])
    for g, e in zip(got[:2], exact[:2]):
        assert_rounded(g.cpu().numpy(), e, abs(L(F(scale))) * np.where(far >= 2.0 ** 45, L(2) ** -34, L(2) ** -44))
    for g, e in zip(got[2:], exact[2:]):
        assert_bound(g.cpu().numpy(), e)


@pytest.mark.parametrize("u", [2.0 ** -30, 2.0 ** -53])
def test_tables_of_finer_models(tao, u):
    """Roundoffs far below binary32's: the angle's own rounding in binary64 would be as large as E."""
    m = tao.FpModel(u=u)
    p = np.array([0, 1, 5, 1001, 70001, 2 ** 24 + 1, 2 ** 31 - 1, 2 ** 40 + 1])
    assert_tables_closely(tao, p, frequencies(40, 1e4), 1.1, m)
    assert_tables_closely(tao, p, frequencies(40, 1e4), 1.0, m)


def test_tables_beyond_their_range(tao):
    f = np.array([1.0, np.inf, np.nan, 3e38, -np.inf, 2.0 ** 50, 2.0 ** 49], F)
    c, s, tc, ts = (t.cpu().numpy() for t in tao.tao_bound_rope_tables(*cuda(f, np.array([1, 2]))))
    for t in (c, s, tc, ts):
        assert np.array_equal(np.isnan(t), [[False, True, True, True, True, True, False], [False, True, True, True, True, True, True]])


@pytest.mark.parametrize("model", [dict(mode=1, lam=4.0), dict(u=2.0 ** -11), dict(c_sin=1.0, c_cos=9.0), dict(c_sin=0.0, c_cos=0.0)])
def test_table_models(tao, model):
    p, f = np.array([0, 1, 5, 1000, 3001, 70000]), frequencies(40, 1e4)
    m = tao.FpModel(**model)
    assert_tables(tao.tao_bound_rope_tables(*cuda(f, p), scale=1.1, model=m), p, f, 1.1, m)


@pytest.mark.parametrize("model,scale", [(dict(c_sin=0.0, c_cos=0.0), 1.0), (dict(c_sin=4.0, c_cos=0.0), 1.0), (dict(c_sin=0.0, c_cos=0.0, u=2.0 ** -11), 1.0), (dict(u=2.0 ** -40), 2.0 ** -40),
                                         (dict(c_sin=1e-20, c_cos=1e-20, u=2.0 ** -40), 2.0 ** -40), (dict(c_sin=1e4, c_cos=0.0), 2.0 ** -100), (dict(), 2.0 ** -120), (dict(c_cos=0.0), 1e30)])
def test_table_bounds_next_to_nothing(tao, model, scale):
    """Angles next to 0 under models and amplitudes that leave hardly any bound: its terms, or it, fall below binary32's smallest normal numbers."""
    rng = np.random.default_rng(5)
    f = np.concatenate([2.0 ** rng.uniform(-75, -20, 400), 2.0 ** -np.arange(40, 62), [1.0, 0.1, 3e-7, 1e-30, 0.0]]).astype(F)
    p = np.array([0, 1, 3, 1001, 70001])
    m = tao.FpModel(**model)
    assert_tables(tao.tao_bound_rope_tables(*cuda(f, p), scale=scale, model=m), p, f, scale, m)


def test_tables_in_part(tao):
    f = cuda(frequencies(8))[0]
    whole = tao.tao_bound_rope_tables(f, npos=9)
    c, s, none, none2 = tao.tao_bound_rope_tables(f, npos=9, with_tau=False)
    assert none is None and none2 is None and torch.equal(c, whole[0]) and torch.equal(s, whole[1])
    only = torch.full((9, 8), 7.0, device="cuda")
    assert tao.lib().tao_bound_rope_tables(None, f.data_ptr(), 1.0, None, None, None, only.data_ptr(), 9, 8, None, tao._stream()) == 0
    assert torch.equal(only, whole[3])
    for npos, half in ((0, 8), (4, 0)):
        assert tao.tao_bound_rope_tables(cuda(frequencies(half))[0], npos=npos)[0].shape == (npos, half)


@pytest.mark.parametrize("npos,half", [(1, 1), (1, 2), (1, 3), (2, 3), (5, 1), (7, 5), (3, 7), (129, 63), (2000, 3), (11, 130), (8323, 63), (174763, 3), (524289, 1), (262145, 2)])
@pytest.mark.parametrize("at", [0, 1])
def test_tables_of_any_length(tao, npos, half, at):
    """Rows that are no whole vectors, with what lies before and behind the tables left as it was, from aligned and other addresses, in both kernels; positions that end where their memory ends."""
    store = torch.empty(20 << 20, dtype=torch.uint8, device="cuda")
    p = np.random.default_rng(npos + half).integers(0, 100000, npos)
    pd = store[len(store) - p.nbytes:].view(torch.int64).copy_(torch.from_numpy(p))
    f = frequencies(half, 1e4)
    whole = [torch.full((npos * half + 8,), 7.0, device="cuda") for _ in range(4)]
    views = [w[at:at + npos * half].view(npos, half) for w in whole]
    got = tao.tao_bound_rope_tables(cuda(f)[0], pd, cos=views[0], sin=views[1], tau_cos=views[2], tau_sin=views[3])
    rows = np.arange(npos) if npos < 3000 else np.unique(np.concatenate([np.arange(40), np.arange(npos - 700, npos), np.random.default_rng(0).integers(0, npos, 500)]))
    assert_tables([t[torch.from_numpy(rows).cuda()] for t in got], p[rows], f)
    for w in whole:
        assert bool((w[:at] == 7).all()) and bool((w[at + npos * half:] == 7).all())


def test_tables_that_are_long(tao):
    f = frequencies(64)
    got = tao.tao_bound_rope_tables(cuda(f)[0], npos=131072)
    rows = np.array([0, 1, 255, 4097, 65535, 99991, 131071])
    assert_tables([t[torch.from_numpy(rows).cuda()] for t in got], rows, f)


# ------------------------------------------------------------------ heads

def heads(T, H, d, rot, npos=None, seed=0, errors=False, norm=True, heads_k=0):
    rng = np.random.default_rng(seed + T * 7 + H * 3 + d + rot)
    npos = npos or max(1, T // 2)
    x = (rng.normal(0, 1, (T, H, d)) * np.exp(rng.normal(0, 2, (T, H, 1)))).astype(F)
    c, s = (rng.uniform(-1, 1, (npos, rot // 2)).astype(F) for _ in range(2))
    k = dict(positions=rng.integers(0, npos, T))
    if errors:
        k["tau_cos"], k["tau_sin"] = (rng.uniform(0, 1e-4, (npos, rot // 2)).astype(F) for _ in range(2))
    if norm:
        k["gamma_q"] = rng.normal(1, 0.3, d).astype(F)
        k["gamma_k"] = rng.normal(-1, 0.3, d).astype(F) if heads_k else None
    return x, c, s, dict(k, norm=norm, heads_k=heads_k)


def both(tao, x, c, s, k, device_x=None, model=None, **more):
    """The library's (y, tau) and the oracle's."""
    e = rotary.norm_rope(x, c, s, 2 * c.shape[1], model=model, **k, **more)
    g = dict(k)
    g["norm"] = tao.NORM_RMSNORM if g["norm"] else tao.NORM_NONE
    g["gamma"] = g.pop("gamma_q", None)
    g = {n: cuda(v)[0] if isinstance(v, np.ndarray) else v for n, v in g.items()}
    got = tao.tao_bound_norm_rope(cuda(x)[0] if device_x is None else device_x, *cuda(c, s), model=model, **g, **more)
    return got, e, g


def assert_heads(got, e, x, rot, what=""):
    y, tau = (t.cpu().numpy() for t in got)
    # what the two products of a pair lose in binary64
    size = np.abs(e[0]).max(axis=-1, keepdims=True, initial=0)
    assert_rounded(y, e[0], np.where(np.isfinite(size), size, 0) * L(2) ** -46, what)
    assert_bound(tau, e[1], what)


SHAPES = [(1, 1, 2, 2), (1, 40, 128, 128), (3, 2, 8, 8), (5, 3, 16, 8), (7, 5, 64, 32), (9, 2, 64, 0), (4, 3, 90, 26), (6, 7, 33, 32), (2, 3, 1, 0), (11, 2, 256, 256),
          (3, 4, 80, 80), (5, 2, 96, 48), (2, 2, 320, 320), (3, 1, 1000, 500), (2, 2, 4100, 4096), (130, 9, 24, 24), (300, 6, 128, 64), (17, 3, 40, 16), (2, 3, 512, 512), (3, 5, 72, 8)]


@pytest.mark.parametrize("T,H,d,rot", SHAPES)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("norm", [False, True])
def test_heads(tao, T, H, d, rot, interleaved, norm):
    x, c, s, k = heads(T, H, d, rot, norm=norm, errors=T % 2 == 1, heads_k=H // 3)
    got, e, _ = both(tao, x, c, s, k, interleaved=interleaved)
    assert_heads(got, e, x, rot)


@pytest.mark.parametrize("d,rot", [(128, 128), (64, 16), (30, 10)])
def test_without_positions_and_gains(tao, d, rot):
    x, c, s, k = heads(13, 3, d, rot, npos=5)
    k.update(positions=None, gamma_q=None)
    got, e, _ = both(tao, x, c, s, k)
    assert_heads(got, e, x, rot)
    x, c, s, k = heads(13, 5, d, rot, heads_k=2)
    for drop in ("gamma_q", "gamma_k"):
        got, e, _ = both(tao, x, c, s, dict(k, **{drop: None}))
        assert_heads(got, e, x, rot)


@pytest.mark.parametrize("d,rot,norm", [(128, 128, True), (128, 64, False), (40, 24, True), (31, 12, True)])
def test_strides_of_fused_projections(tao, d, rot, norm):
    """Heads inside wider rows, heads before tokens, and rows that begin at any address; what lies between holds NaN and must not count."""
    x, c, s, k = heads(6, 5, d, rot, norm=norm, heads_k=2)
    plain, e, _ = both(tao, x, c, s, k)
    for at, extra, wide in ((0, 0, 3), (1, 3, 1), (4, 8, 0), (2, 1, 2)):
        store = torch.full((at + 6 * ((5 + wide) * (d + extra)) + 8,), float("nan"), device="cuda")
        view = store[at:at + 6 * (5 + wide) * (d + extra)].view(6, 5 + wide, d + extra)[:, :5, :d]
        view.copy_(torch.from_numpy(x))
        got, _, _ = both(tao, x, c, s, k, device_x=view)
        assert torch.equal(got[0], plain[0]) and torch.equal(got[1], plain[1])
    by_head = torch.from_numpy(np.ascontiguousarray(x.transpose(1, 0, 2))).cuda().transpose(0, 1)
    got, _, _ = both(tao, x, c, s, k, device_x=by_head)
    assert torch.equal(got[0], plain[0]) and torch.equal(got[1], plain[1])
    shared = torch.from_numpy(x[:, :1]).cuda().expand(6, 5, d)              # one head that all read
    got, e, _ = both(tao, np.repeat(x[:, :1], 5, axis=1), c, s, k, device_x=shared)
    assert_heads(got, e, x, rot)


@pytest.mark.parametrize("d,rot", [(64, 64), (18, 6)])
@pytest.mark.parametrize("by_head", [False, True])
def test_outputs_keep_what_lies_between_them(tao, d, rot, by_head):
    T, H = 5, 3
    x, c, s, k = heads(T, H, d, rot)
    plain, _, g = both(tao, x, c, s, k)
    ldyt, ldyh = (d + 3, T * (d + 3) + 5) if by_head else (H * (d + 4) + 7, d + 4)
    n = T * ldyt + H * ldyh + d
    y, tau = torch.full((n,), 7.0, device="cuda"), torch.full((n,), 7.0, device="cuda")
    xd, cd, sd = cuda(x, c, s)
    rc = tao.lib().tao_bound_norm_rope(1, xd.data_ptr(), g["gamma"].data_ptr(), None, 1e-6, cd.data_ptr(), sd.data_ptr(), None, None, g["positions"].data_ptr(), y.data_ptr(),
                                       tau.data_ptr(), T, H, 0, d, rot, len(c), H * d, d, ldyt, ldyh, 0, None, tao._stream())
    assert rc == 0
    for whole, part in ((y, plain[0]), (tau, plain[1])):
        view = whole.as_strided((T, H, d), (ldyt, ldyh, 1))
        assert torch.equal(view, part)
        view.fill_(7.0)
        assert bool((whole == 7.0).all())


def test_positions_outside_the_tables(tao):
    for d, rot in ((128, 64), (20, 8)):
        x, c, s, k = heads(9, 2, d, rot, npos=6)
        k["positions"][[1, 4, 5, 8]] = [-1, 6, 2 ** 40, -2 ** 63]
        got, e, g = both(tao, x, c, s, k)
        assert np.isnan(e[0][[1, 4, 5, 8], :, :rot]).all() and not np.isnan(e[0][:, :, rot:]).any()
        assert_heads(got, e, x, rot)
        pf = tao.tao_bound_check_norm_rope(cuda(x)[0], *cuda(c, s), got[0].clone(), **g)
        assert pf["violations"] == 4 * 2 * rot and pf["nan_count"] == 4 * 2 * rot


@pytest.mark.parametrize("d,rot", [(128, 64), (21, 10)])
@pytest.mark.parametrize("norm", [False, True])
def test_values_that_are_no_ordinary_numbers(tao, d, rot, norm):
    x, c, s, k = heads(14, 2, d, rot, npos=14, norm=norm, errors=True)
    k["positions"] = np.arange(14)
    x[0, 0, 1], x[1, 0, d - 1], x[2, 1, 0] = np.inf, -np.inf, np.nan
    x[3], x[4], x[5], x[6] = 0, 1e-42, 3e38, 1e-30
    c[7, 1], s[8, 0], k["tau_cos"][9, 0], k["tau_sin"][10, 1], c[11, 2] = np.nan, np.inf, np.nan, np.inf, 0
    if norm:
        k["gamma_q"][[1, 2, 3]] = [np.inf, np.nan, 0]
    got, e, g = both(tao, x, c, s, k)
    y, tau = (t.cpu().numpy() for t in got)
    assert_bound(tau, e[1])
    fine = np.isfinite(e[1])
    assert_rounded(np.where(fine, y, 0), np.where(fine, e[0], 0), np.where(fine, np.abs(np.where(fine, e[0], 0)).max(axis=-1, keepdims=True), 0) * L(2) ** -46)
    pf = tao.tao_bound_check_norm_rope(cuda(x)[0], *cuda(c, s), got[0].clone(), **g)
    assert_profile_equal(pf, oracle.check_and_profile(y, y, tau))
    assert pf["violations"] >= (~fine).sum()
    zero_eps, e, _ = both(tao, x, c, s, k, eps=0.0)           # rows of zeros have no norm then
    assert_bound(zero_eps[1].cpu().numpy(), e[1])


@pytest.mark.parametrize("model", [dict(mode=1, lam=4.0), dict(flags=1), dict(u=2.0 ** -11), dict(flags=1, u=2.0 ** -20, c_rsqrt=5.0, c_div=3.0)])
@pytest.mark.parametrize("d,rot", [(64, 64), (50, 20)])
def test_head_models(tao, model, d, rot):
    x, c, s, k = heads(8, 3, d, rot, errors=True)
    x[2] *= F(1e-30)
    got, e, _ = both(tao, x, c, s, k, model=tao.FpModel(**model))
    assert_heads(got, e, x, rot)


def test_one_of_the_two_outputs(tao):
    for d, rot in ((128, 128), (22, 8)):
        x, c, s, k = heads(7, 3, d, rot)
        (y, tau), _, g = both(tao, x, c, s, k)
        a = cuda(x, c, s)
        y1, none = tao.tao_bound_norm_rope(*a, with_tau=False, **g)
        none2, t1 = tao.tao_bound_norm_rope(*a, with_y=False, **g)
        assert none is None and none2 is None and torch.equal(y, y1) and torch.equal(tau, t1)


def test_heads_of_nothing(tao):
    for T, H, d, rot in ((0, 3, 8, 8), (3, 0, 8, 8), (3, 2, 0, 0)):
        x, c, s = torch.empty((T, H, d), device="cuda"), torch.ones((4, rot // 2), device="cuda"), torch.ones((4, rot // 2), device="cuda")
        y, tau = tao.tao_bound_norm_rope(x, c, s)
        assert y.shape == tau.shape == (T, H, d)
        pf = tao.tao_bound_check_norm_rope(x, c, s, torch.empty_like(x))
        assert pf["n"] == 0 and pf["accept"] == 1 and pf["hist"].sum() == 0


CHECKED = [(1, 1, 2, 2), (1, 40, 128, 128), (3, 4, 90, 26), (100, 5, 64, 64), (64, 40, 128, 128), (33, 7, 96, 32), (700, 3, 80, 80), (260, 40, 128, 64), (3, 3, 4100, 16), (2000, 10, 64, 32)]


@pytest.mark.parametrize("T,H,d,rot", CHECKED)
@pytest.mark.parametrize("ref", [False, True])
@pytest.mark.parametrize("norm", [False, True])
def test_check_is_the_streaming_check_of_the_stored_bound(tao, T, H, d, rot, ref, norm):
    x, c, s, k = heads(T, H, d, rot, norm=norm, errors=not norm, heads_k=H // 4)
    g = dict(k, norm=tao.NORM_RMSNORM if norm else tao.NORM_NONE, interleaved=T % 2 == 0)
    g["gamma"] = g.pop("gamma_q", None)
    g = {n: cuda(v)[0] if isinstance(v, np.ndarray) else v for n, v in g.items()}
    a = cuda(x, c, s)
    y, tau = tao.tao_bound_norm_rope(*a, **g)
    r = torch.Generator(device="cuda").manual_seed(T + d)
    f = torch.tensor([0.0, 0.0, 0.5, -0.99, 1.0, 1.01, -3.0, 1e6], device="cuda")[torch.randint(0, 8, y.shape, generator=r, device="cuda")]
    claimed = (y.double() + f.double() * tau.double()).float()
    claimed.view(-1)[0] = float("nan")
    claimed.view(-1)[-1] = float("inf")
    y_ref = (y * (1 + 2.0 ** -23)).contiguous() if ref else None
    for alpha, eps_rel in ((1.0, 1e-12), (2.0, 0.0), (0.0, 1.0)):
        pf = tao.tao_bound_check_norm_rope(*a, claimed, y_ref=y_ref, alpha=alpha, eps_rel=eps_rel, **g)
        other = y if y_ref is None else y_ref
        assert_profile_equal(pf, oracle.check_and_profile(claimed.cpu().numpy(), other.cpu().numpy(), tau.cpu().numpy(), alpha, eps_rel))
    honest = tao.tao_bound_check_norm_rope(*a, y.clone(), **g)
    assert honest["accept"] == 1 and honest["max_rel"] == 0.0 and honest["n"] == T * H * d


@pytest.mark.parametrize("d", [2, 3, 15, 16, 17, 31, 32, 33, 63, 65, 66, 127, 129, 130, 255, 257, 258, 511, 513])
@pytest.mark.parametrize("interleaved", [False, True])
def test_heads_of_any_length(tao, d, interleaved):
    """Lengths at the borders of the lanes that a head has: whole heads rotated, half of them, and none; outputs, bounds and the checks of claims at and around their bounds."""
    for rot in {d // 2 * 2, d // 4 * 2, 0}:
        x, c, s, k = heads(21, 3, d, rot, errors=rot % 4 == 0, heads_k=1)
        got, e, g = both(tao, x, c, s, k, interleaved=interleaved)
        assert_heads(got, e, x, rot)
        y, tau = got
        f = torch.tensor([0.0, 0.5, -0.99, 1.01, 0.0, -3.0], device="cuda")[torch.arange(y.numel(), device="cuda") % 6].view(y.shape)
        claimed = (y.double() + f.double() * tau.double()).float()
        for y_ref in (None, (y * (1 + 2.0 ** -22)).contiguous()):
            pf = tao.tao_bound_check_norm_rope(cuda(x)[0], *cuda(c, s), claimed, y_ref=y_ref, interleaved=interleaved, **g)
            other = y if y_ref is None else y_ref
            assert_profile_equal(pf, oracle.check_and_profile(claimed.cpu().numpy(), other.cpu().numpy(), tau.cpu().numpy(), 1.0, 1e-12))


@pytest.mark.parametrize("d,rot", [(24, 8), (32, 32), (64, 24), (136, 128), (512, 256)])
@pytest.mark.parametrize("errors", [False, True])
def test_vectors_of_neighbouring_pairs(tao, d, rot, errors):
    """Interleaved pairs in whole vectors, some of whose lanes have a rotated vector and one that is not."""
    x, c, s, k = heads(50, 5, d, rot, errors=errors, heads_k=2)
    k["positions"][[3, 40]] = [-1, 10 ** 9]
    got, e, g = both(tao, x, c, s, k, interleaved=True)
    assert_heads(got, e, x, rot)
    pf = tao.tao_bound_check_norm_rope(cuda(x)[0], *cuda(c, s), got[0].clone(), interleaved=True, **g)
    y, tau = (t.cpu().numpy() for t in got)
    assert_profile_equal(pf, oracle.check_and_profile(y, y, tau))


@pytest.mark.parametrize("T,H,d,rot", [(20, 5, 128, 128), (600, 40, 128, 128), (300, 7, 50, 20)])
def test_the_largest_error_among_many(tao, T, H, d, rot):
    """Claims whose largest error is one of many almost as large, the last of a rising row, the first of a falling one, or the only one."""
    x, c, s, k = heads(T, H, d, rot)
    a, g = cuda(x, c, s), dict(gamma=cuda(k["gamma_q"])[0], positions=cuda(k["positions"])[0])
    y, tau = tao.tao_bound_norm_rope(*a, **g)
    v, n = y.double(), y.numel()
    ramp = torch.arange(1, n + 1, device="cuda", dtype=torch.float64).view(y.shape) / n
    one = y.clone()
    one.view(-1)[n // 3] *= 1.5
    for claimed in ((v * (1 + 1e-3)).float(), (v * (1 + 1e-3 * ramp)).float(), (v * (1 + 1e-3 * (1 + 1 / n - ramp))).float(), one, torch.nextafter(y, torch.zeros_like(y)), 0 * y):
        pf = tao.tao_bound_check_norm_rope(*a, claimed, eps_rel=1e-9, **g)
        assert_profile_equal(pf, oracle.check_and_profile(claimed.cpu().numpy(), y.cpu().numpy(), tau.cpu().numpy(), 1.0, 1e-9))


@pytest.mark.parametrize("d,rot", [(128, 128), (30, 12)])
def test_offsets_beyond_32_bits(tao, d, rot):
    """Tokens of x, and of the outputs, so far apart that the last ones lie more than 2^31 elements on."""
    T, H = 5, 2
    x, c, s, k = heads(T, H, d, rot)
    plain, _, g = both(tao, x, c, s, k)
    step = 2 ** 29 + 2 ** 20
    far = torch.empty((T * step,), device="cuda")
    view = far.as_strided((T, H, d), (step, d, 1)).copy_(torch.from_numpy(x))
    got, _, _ = both(tao, x, c, s, k, device_x=view)
    assert torch.equal(got[0], plain[0]) and torch.equal(got[1], plain[1])
    xd, cd, sd = cuda(x, c, s)
    rc = tao.lib().tao_bound_norm_rope(1, xd.data_ptr(), g["gamma"].data_ptr(), None, 1e-6, cd.data_ptr(), sd.data_ptr(), None, None, g["positions"].data_ptr(), far.data_ptr(),
                                       None, T, H, 0, d, rot, len(c), H * d, d, step, d, 0, None, tao._stream())
    assert rc == 0 and torch.equal(view, plain[0])


@pytest.mark.parametrize("T,H,d,rot", [(3, 2, 8, 8), (5, 3, 90, 26), (7, 5, 128, 64), (1, 1, 24, 0), (9, 1, 136, 136)])
def test_operands_that_end_where_their_memory_ends(tao, T, H, d, rot):
    def at_the_end(a):
        store = torch.empty(20 << 20, dtype=torch.uint8, device="cuda")
        return store[len(store) - a.nbytes:].view(torch.from_numpy(a).dtype).view(a.shape).copy_(torch.from_numpy(a))
    x, c, s, k = heads(T, H, d, rot, errors=True)
    plain, _, _ = both(tao, x, c, s, k)
    g = {n: at_the_end(k[n]) for n in ("positions", "tau_cos", "tau_sin")}
    got = tao.tao_bound_norm_rope(at_the_end(x), at_the_end(c), at_the_end(s), gamma=at_the_end(k["gamma_q"]), **g)
    assert torch.equal(got[0], plain[0]) and torch.equal(got[1], plain[1])
    p, f = k["positions"], frequencies(rot // 2)
    for a, b in zip(tao.tao_bound_rope_tables(*cuda(f, p)), tao.tao_bound_rope_tables(at_the_end(f), at_the_end(p))):
        assert torch.equal(a, b)


def test_refusals_of_the_binding(tao):
    x, c, s, k = heads(4, 3, 16, 16, npos=4)
    xd, cd, sd = cuda(x, c, s)
    gamma, pos = cuda(k["gamma_q"], k["positions"])
    call, check, tables = tao.tao_bound_norm_rope, tao.tao_bound_check_norm_rope, tao.tao_bound_rope_tables
    for bad in (lambda: call(xd.double(), cd, sd), lambda: call(xd.cpu(), cd, sd), lambda: call(xd, cd, sd, positions=pos.int()), lambda: check(xd, cd, sd, None),
                lambda: tables(gamma.double(), npos=3), lambda: tables(gamma, pos.float()), lambda: call(xd, cd, sd, gamma=gamma.half())):
        with pytest.raises(TypeError):
            bad()
    for bad in (lambda: call(xd[0], cd, sd), lambda: call(xd, cd, sd[:, :7].contiguous()), lambda: call(xd, cd, None), lambda: call(xd, cd, sd, gamma=gamma[:8]),
                lambda: call(xd, cd, sd, gamma_k=gamma), lambda: call(xd, cd, sd, heads_k=4), lambda: call(xd, cd, sd, heads_k=-1), lambda: call(xd, cd, sd, positions=pos[:3]),
                lambda: call(xd, cd, sd, tau_cos=cd), lambda: call(xd[:, :, ::2], cd, sd), lambda: call(xd, cd, sd, y=torch.empty((4, 3, 15), device="cuda")),
                lambda: call(xd, cd, sd, with_y=False, with_tau=False), lambda: check(xd, cd, sd, xd[:3].contiguous()), lambda: check(xd, cd, sd, xd, ws=torch.empty(64, dtype=torch.uint8, device="cuda")),
                lambda: tables(gamma), lambda: tables(gamma, pos, npos=3), lambda: tables(gamma[None], npos=3), lambda: tables(gamma, npos=3, cos=torch.empty((3, 15), device="cuda"))):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: call(xd, cd, sd, norm=tao.NORM_LAYERNORM), lambda: call(xd, cd, sd, norm=tao.NORM_NONE, gamma=gamma), lambda: call(xd, cd.repeat(1, 2), sd.repeat(1, 2)),
                lambda: tables(gamma, npos=-1), lambda: check(xd, cd, sd, xd, alpha=-1.0), lambda: call(xd, cd, sd, eps=-1.0)):
        with pytest.raises((tao.TaoError, RuntimeError)):
            bad()


# ------------------------------------------------------------------ more heads, and longer tables, than a launch has lanes for at once

@pytest.mark.parametrize("T,d,rot,interleaved", [(70001, 264, 264, False), (70001, 264, 136, True), (131201, 136, 128, False), (262301, 128, 128, False), (524401, 64, 32, False), (1048701, 32, 32, True), (70001, 258, 258, False),
                                                 (70001, 130, 66, False), (1048701, 14, 6, True), (66001, 520, 512, False)])
def test_more_heads_than_a_launch_has_lanes_for(tao, T, d, rot, interleaved):
    """Every kernel's lanes take a second head, in a last trip that is not whole: the first heads, those next to the seam and the last ones against the oracle; then the check of claims that leave their bounds here and there."""
    g = torch.Generator(device="cuda").manual_seed(d)
    npos = 501
    x = torch.randn((T, 1, d), generator=g, device="cuda")
    c, s = (torch.rand((npos, rot // 2), generator=g, device="cuda") * 2 - 1 for _ in range(2))
    gamma = 1 + 0.1 * torch.randn(d, generator=g, device="cuda")
    positions = torch.randint(0, npos, (T,), generator=g, device="cuda")
    k = dict(gamma=gamma, positions=positions, interleaved=interleaved)
    y, tau = tao.tao_bound_norm_rope(x, c, s, **k)
    lanes = next(n for n in (4, 8, 16, 32, 64) if d <= 8 * n or n == 64) if d % 8 == 0 and d <= 512 else next(n for n in (4, 8, 16, 32, 64) if d <= 4 * n or n == 64)
    seam = 16384 * (256 // lanes)
    assert seam < T < 2 * seam
    rows = torch.cat([torch.arange(40), torch.arange(seam - 40, seam + 40), torch.arange(T - 40, T), torch.randint(0, T, (100,))])
    assert int(rows.max()) < T
    rows = rows.cuda()
    e = rotary.norm_rope(x[rows].cpu().numpy(), c.cpu().numpy(), s.cpu().numpy(), rot, gamma_q=gamma.cpu().numpy(), positions=positions[rows].cpu().numpy(), interleaved=interleaved)
    assert_heads((y[rows], tau[rows]), e, None, rot)
    f = torch.tensor([0.0, 0.0, 0.5, -0.9, 0.0], device="cuda")[torch.arange(y.numel(), device="cuda") % 5].view(y.shape)
    claimed = (y.double() + f.double() * tau.double()).float()
    claimed[[0, seam - 1, seam, T - 1], 0, 1] += 3 * tau[[0, seam - 1, seam, T - 1], 0, 1]
    pf = tao.tao_bound_check_norm_rope(x, c, s, claimed, **k)
    assert pf["violations"] == 4
    assert_profile_equal(pf, oracle.check_and_profile(claimed.cpu().numpy(), y.cpu().numpy(), tau.cpu().numpy(), 1.0, 1e-12))


@pytest.mark.parametrize("npos,half,at", [(262209, 64, 0), (270001, 63, 0), (70001, 63, 1)])
def test_longer_tables_than_a_launch_has_lanes_for(tao, npos, half, at):
    """Vectors of whole rows, vectors over the ends of rows, and elements from an address that fits no vector."""
    f, n = frequencies(half), npos * half
    whole = [torch.full((n + 8,), 7.0, device="cuda") for _ in range(4)]
    views = [w[at:at + n].view(npos, half) for w in whole]
    got = tao.tao_bound_rope_tables(cuda(f)[0], npos=npos, cos=views[0], sin=views[1], tau_cos=views[2], tau_sin=views[3])
    seam = 16384 * 256 * (1 if at else 4) // half
    assert seam < npos < 2 * seam
    rows = np.concatenate([np.arange(20), np.arange(seam - 20, seam + 20), np.arange(npos - 20, npos), np.random.default_rng(1).integers(0, npos, 60)])
    assert rows.max() < npos
    assert_tables([t[torch.from_numpy(rows).cuda()] for t in got], rows, f)
    for w in whole:
        assert bool((w[:at] == 7).all()) and bool((w[at + n:] == 7).all())
