"""Channels-last GroupNorm with an activation against its oracle: outputs to their last rounding, bounds one-sided within 1e-6, profiles
equal to the streaming check of the stored output and bound."""
import numpy as np
import pytest
import torch

import oracle
from oracle import groupnorm_act as gn
from opmap import assert_profile_equal

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tao():
    import paper_2510_16028_amd as t
    return t


def kinds(tao):
    return {gn.NONE: tao.ACT_EXACT, gn.RELU: tao.ACT_RELU, gn.SILU: tao.ACT_SILU}


def inputs(B, P, C, seed=0, scale=1.0, shift=0.0):
    rng = np.random.default_rng(seed)
    x = (rng.normal(shift, scale, (B, P, C)) + rng.normal(0, scale / 2, (B, 1, C))).astype(np.float32)
    return x, rng.normal(1, 0.3, C).astype(np.float32), rng.normal(0, 0.5, C).astype(np.float32)


def cuda(*arrays):
    return [None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda() for a in arrays]


def assert_outputs(y, tau, ye, te, E, act):
    """y: the last rounding is half a step, 2^-24 |y|, and what precedes it in binary64 lies far below 2^-20 tau (which holds several 2^-24 of
    every intermediate).  tau: at or above the formula's value and within 1e-6 of it (ReLU: of E); one step where it is subnormal."""
    L = np.longdouble
    y, tau = y.cpu().numpy().astype(L), tau.cpu().numpy().astype(L)
    assert np.array_equal(np.isnan(tau), np.isnan(te)) and np.array_equal(np.isnan(y), np.isnan(ye))
    ok = ~np.isnan(ye)
    assert (np.abs(y - ye)[ok] <= (np.abs(ye) * L(2) ** -24 * (1 + L(2) ** -10) + np.nan_to_num(te) * L(2) ** -20 + L(2) ** -149)[ok]).all()
    ok = ~np.isnan(te)
    assert (tau >= te * (1 - L(2) ** -58))[ok].all(), float((tau / te)[ok & (te > 0)].min())
    room = te * (1 + L(1e-6)) + (E * L(1e-6) if act == gn.RELU else 0) + L(2) ** -149
    assert (tau <= room)[ok].all(), float((tau / np.maximum(te, 1e-300))[ok].max() - 1)


SHAPES = [(1, 1, 4, 1), (1, 1, 4, 2), (2, 3, 5, 5), (1, 7, 6, 3), (2, 64, 1280, 32), (3, 50, 40, 8), (1, 300, 37, 1), (2, 256, 320, 32), (1, 1024, 128, 32),
          (4, 33, 96, 96), (1, 5000, 8, 2), (2, 500, 516, 4), (1, 100, 2048, 1), (1, 20, 4100, 4), (1, 9000, 12, 1), (40, 10, 64, 16), (300, 4, 12, 3), (1, 17, 1030, 515), (1, 3, 700, 700),
          (2, 2500, 320, 32), (1, 1300, 1030, 103), (520, 1, 12, 3), (8, 100, 256, 64), (1, 513, 2052, 513)]


@pytest.mark.parametrize("B,P,C,groups", SHAPES)
@pytest.mark.parametrize("act", [gn.NONE, gn.RELU, gn.SILU])
def test_outputs_and_bounds(tao, B, P, C, groups, act):
    x, gamma, beta = inputs(B, P, C, P + C)
    y, tau = tao.tao_bound_groupnorm_act(*cuda(x), groups, *cuda(gamma, beta), 1e-5, act=kinds(tao)[act])
    assert_outputs(y, tau, *gn.groupnorm_act(act, x, groups, gamma, beta, 1e-5), act)


@pytest.mark.parametrize("scale,shift", [(1e-4, 3.0), (50.0, -200.0), (1e-12, 0.0), (1e15, 1e15), (1e-3, 0.0)])
@pytest.mark.parametrize("act", [gn.NONE, gn.RELU, gn.SILU])
def test_ranges(tao, scale, shift, act):
    x, gamma, beta = inputs(2, 40, 24, 3, scale, shift)
    gamma[:4] *= 40                                          # arguments far out on both sides of the activation
    y, tau = tao.tao_bound_groupnorm_act(*cuda(x), 4, *cuda(gamma, beta), 1e-6, act=kinds(tao)[act])
    assert_outputs(y, tau, *gn.groupnorm_act(act, x, 4, gamma, beta, 1e-6), act)


@pytest.mark.parametrize("act", [gn.NONE, gn.RELU, gn.SILU])
def test_groups_without_a_bound_and_numbers_that_are_none(tao, act):
    x, gamma, beta = inputs(3, 30, 16, 6)
    x[0, :, :4] = 2.5                                        # constant and no eps: no bound
    x[1, 4, 5] = np.nan; x[1, 5, 9] = np.inf; x[2, 0, 15] = -np.inf
    gamma[7] = 0.0
    y, tau = tao.tao_bound_groupnorm_act(*cuda(x), 4, *cuda(gamma, beta), 0.0, act=kinds(tao)[act])
    _, te, _ = gn.groupnorm_act(act, x, 4, gamma, beta, 0.0)
    t = tau.cpu().numpy()
    none = np.isnan(te.astype(np.float64))
    assert none[0, :, :4].all() and none[1, :, 4:12].all() and none[2, :, 12:].all() and none.sum() == 30 * 4 * 4
    assert np.array_equal(np.isnan(t), none)
    assert (t[~none] >= te[~none] * (1 - np.longdouble(2) ** -58)).all()
    pf = tao.tao_bound_check_groupnorm_act(*cuda(x), y, 4, *cuda(gamma, beta), 0.0, act=kinds(tao)[act])
    assert_profile_equal(pf, oracle.check_and_profile(y.cpu().numpy(), y.cpu().numpy(), t))
    assert pf["violations"] == none.sum()


def test_without_gamma_and_beta_and_one_of_the_two_outputs(tao):
    x, gamma, beta = inputs(2, 70, 48, 2)
    xd, gd, bd = cuda(x, gamma, beta)
    for g, b in ((None, None), (gd, None), (None, bd)):
        y, tau = tao.tao_bound_groupnorm_act(xd, 6, g, b)
        assert_outputs(y, tau, *gn.groupnorm_act(gn.SILU, x, 6, gamma if g is not None else None, beta if b is not None else None, 1e-5), gn.SILU)
        y1, none = tao.tao_bound_groupnorm_act(xd, 6, g, b, with_tau=False)
        none2, t1 = tao.tao_bound_groupnorm_act(xd, 6, g, b, with_y=False)
        assert none is None and none2 is None and torch.equal(y, y1) and torch.equal(tau, t1)


@pytest.mark.parametrize("C,ld,at", [(8, 20, 0), (8, 20, 3), (12, 16, 4), (6, 11, 2), (64, 128, 64)])
def test_slices_of_channels(tao, C, ld, at):
    """A part of the channels of wider features, at any address: pixels further apart than they are long."""
    whole, _, _ = inputs(2, 36, ld, 1)
    x = whole.reshape(2, 6, 6, ld)[..., at:at + C]
    gamma, beta = inputs(1, 1, C, 5)[1:]
    xd = torch.from_numpy(whole.reshape(2, 6, 6, ld)).cuda()[..., at:at + C]
    y, tau = tao.tao_bound_groupnorm_act(xd, 2, *cuda(gamma, beta))
    ye, te, E = (t.reshape(2, 6, 6, C) for t in gn.groupnorm_act(gn.SILU, x.reshape(2, 36, C), 2, gamma, beta))
    assert_outputs(y, tau, ye, te, E, gn.SILU)
    claimed = torch.where(torch.rand_like(y) < 0.3, y + 3 * tau, y)
    pf = tao.tao_bound_check_groupnorm_act(xd, claimed, 2, *cuda(gamma, beta))
    assert_profile_equal(pf, oracle.check_and_profile(claimed.cpu().numpy(), y.cpu().numpy(), tau.cpu().numpy()))


@pytest.mark.parametrize("P,C,groups,pad,at", [(900, 12, 2, 5, 3), (2500, 10, 2, 1, 1), (1200, 7, 1, 2, 0), (40, 36, 6, 4, 4)])
def test_pixels_further_apart_than_they_are_long(tao, P, C, groups, pad, at):
    """The same bits from padded pixels as from dense ones, and what lies between those of the results stays as it was."""
    x, gamma, beta = inputs(2, P, C, 9)
    xd, gd, bd = cuda(x, gamma, beta)
    y, tau = tao.tao_bound_groupnorm_act(xd, groups, gd, bd)
    ld = C + pad
    room = torch.full((2, P, ld), 7.0, device="cuda")
    room[..., at:at + C] = xd
    outs = [torch.full((2 * P * ld,), 9.0, device="cuda") for _ in range(2)]
    L, ws = tao.lib(), torch.empty(max(256, tao.tao_groupnorm_act_workspace_bytes(2, P, C, groups)), dtype=torch.uint8, device="cuda")
    place = lambda t: t.data_ptr() + 4 * at
    rc = L.tao_bound_groupnorm_act(tao.ACT_SILU, place(room), gd.data_ptr(), bd.data_ptr(), 1e-5, place(outs[0]), place(outs[1]), 2, P, C, groups, ld, ld, None,
                                   ws.data_ptr(), ws.numel(), torch.cuda.current_stream().cuda_stream)
    assert rc == tao.OK
    for out, dense in zip(outs, (y, tau)):
        out = out.view(2, P, ld)
        assert torch.equal(out[..., at:at + C], dense)
        assert bool((out[..., :at] == 9).all()) and bool((out[..., at + C:] == 9).all())


@pytest.mark.parametrize("P", [300, 700000])
def test_offsets_beyond_32_bits(tao, P):
    """Eight channels out of so many that the last pixel lies more than 2^31 elements on."""
    ld = 2 ** 31 // P + 64
    x = torch.empty((1, P, ld), device="cuda")[..., 40:48].normal_()
    y, tau = tao.tao_bound_groupnorm_act(x, 2)
    y2, tau2 = tao.tao_bound_groupnorm_act(x.contiguous(), 2)
    assert torch.equal(y, y2) and torch.equal(tau, tau2)


def test_channels_last_memory_format_is_taken_as_it_is(tao):
    x = torch.randn((2, 32, 7, 9), device="cuda").contiguous(memory_format=torch.channels_last)
    y, _ = tao.tao_bound_groupnorm_act(x.permute(0, 2, 3, 1), 8)
    expect = torch.nn.functional.silu(torch.nn.functional.group_norm(x.double(), 8)).permute(0, 2, 3, 1)
    assert (y.double() - expect).abs().max() < 1e-5


def test_models(tao):
    x, gamma, beta = inputs(2, 200, 24, 8)
    for model in (dict(mode=1), dict(u=2.0 ** -20), dict(c_exp=4.0, c_rsqrt=3.0, c_div=1.0)):
        m = tao.FpModel(**model)
        for act in (gn.NONE, gn.RELU, gn.SILU):
            y, tau = tao.tao_bound_groupnorm_act(*cuda(x), 3, *cuda(gamma, beta), act=kinds(tao)[act], model=m)
            assert_outputs(y, tau, *gn.groupnorm_act(act, x, 3, gamma, beta, 1e-5, model=m), act)


CHECKED = SHAPES + [(2, 4096, 64, 32), (600, 3, 20, 5), (1, 30000, 10, 2)]


@pytest.mark.parametrize("B,P,C,groups", CHECKED)
@pytest.mark.parametrize("ref", [False, True])
def test_check_is_the_streaming_check_of_the_stored_bound(tao, B, P, C, groups, ref):
    act = (gn.NONE, gn.RELU, gn.SILU)[(B + P + C) % 3]
    x, gamma, beta = inputs(B, P, C, B + P + C)
    a = cuda(x)[0], groups, *cuda(gamma, beta)
    y, tau = tao.tao_bound_groupnorm_act(*a, act=kinds(tao)[act])
    g = torch.Generator(device="cuda").manual_seed(P)
    f = torch.tensor([0.0, 0.0, 0.5, -0.99, 1.0, 1.01, -3.0, 1e6], device="cuda")[torch.randint(0, 8, y.shape, generator=g, device="cuda")]
    claimed = (y.double() + f.double() * tau.double()).float()
    claimed.view(-1)[0] = float("nan")
    claimed.view(-1)[-1] = float("inf")
    y_ref = (y * (1 + 2.0 ** -23)).contiguous() if ref else None
    for alpha, eps_rel in ((1.0, 1e-12), (2.0, 0.0)):
        pf = tao.tao_bound_check_groupnorm_act(a[0], claimed, *a[1:], act=kinds(tao)[act], y_ref=y_ref, alpha=alpha, eps_rel=eps_rel)
        other = y if y_ref is None else y_ref
        assert_profile_equal(pf, oracle.check_and_profile(claimed.cpu().numpy(), other.cpu().numpy(), tau.cpu().numpy(), alpha, eps_rel))


def sets_of_errors(y):
    """Claims whose largest error is one of many almost as large, the last of a rising row, the first of a falling one, or the only one."""
    n = y.numel()
    ramp = torch.arange(1, n + 1, device="cuda", dtype=torch.float64).view(y.shape) / n
    one = y.clone()
    one.view(-1)[n // 3] *= 1.5
    d = y.double()
    return [(d * (1 + 1e-3)).float(), (d * (1 + 1e-3 * ramp)).float(), (d * (1 + 1e-3 * (1 + 1 / n - ramp))).float(), one, torch.nextafter(y, torch.zeros_like(y)), 0 * y]


@pytest.mark.parametrize("B,P,C,groups", [(2, 64, 320, 32), (1, 3000, 64, 8), (1, 1500, 35, 5)])
def test_the_largest_error_among_many(tao, B, P, C, groups):
    x, gamma, beta = inputs(B, P, C, 4)
    a = cuda(x), groups, cuda(gamma, beta)
    y, tau = tao.tao_bound_groupnorm_act(*a[0], groups, *a[2])
    for claimed in sets_of_errors(y):
        pf = tao.tao_bound_check_groupnorm_act(*a[0], claimed, groups, *a[2], eps_rel=1e-9)
        assert_profile_equal(pf, oracle.check_and_profile(claimed.cpu().numpy(), y.cpu().numpy(), tau.cpu().numpy(), 1.0, 1e-9))


def test_nothing_to_do(tao):
    for shape in ((0, 4, 4, 8), (2, 0, 4, 8)):
        x = torch.empty(shape, device="cuda")
        y, tau = tao.tao_bound_groupnorm_act(x, 4)
        assert y.shape == x.shape == tau.shape
        pf = tao.tao_bound_check_groupnorm_act(x, torch.empty(shape, device="cuda"), 4)
        assert pf["n"] == 0 and pf["accept"] == 1 and pf["hist"].sum() == 0


def test_refusals_of_the_binding(tao):
    x = torch.randn((2, 5, 8), device="cuda")
    for bad in (lambda: tao.tao_bound_groupnorm_act(x.half(), 2), lambda: tao.tao_bound_groupnorm_act(x.cpu(), 2),
                lambda: tao.tao_bound_check_groupnorm_act(x, None, 2)):
        with pytest.raises(TypeError):
            bad()
    for bad in (lambda: tao.tao_bound_groupnorm_act(x, 2, x[0, 0, :7]), lambda: tao.tao_bound_groupnorm_act(x.transpose(1, 2), 5),
                lambda: tao.tao_bound_groupnorm_act(x[0, 0], 2), lambda: tao.tao_bound_groupnorm_act(x, 2, y=x[..., :4]),
                lambda: tao.tao_bound_groupnorm_act(x, 2, with_y=False, with_tau=False), lambda: tao.tao_bound_check_groupnorm_act(x, x[:1], 2),
                lambda: tao.tao_bound_groupnorm_act(torch.randn((2, 6, 5, 8), device="cuda")[:, :3], 2)):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: tao.tao_bound_groupnorm_act(x, 3), lambda: tao.tao_bound_groupnorm_act(x, 2, act=tao.ACT_GELU_TANH), lambda: tao.tao_bound_groupnorm_act(x, 2, eps=-1.0)):
        with pytest.raises(tao.TaoError):
            bad()


@pytest.mark.parametrize("act", [gn.NONE, gn.SILU])
def test_a_group_next_to_one_that_almost_has_no_bound(tao, act):
    """The smallest eps with which the first group's variance stays apart from its error: its bound grows by a step of eps a millionfold and may
    take a margin for that; its neighbour, of which a thread has a channel too, keeps its own."""
    x, gamma, beta = inputs(1, 500, 10, 8)
    x[..., :5] = (30000 + x[..., :5] * 0.01).astype(np.float32)
    lo, hi = 0, int(np.float32(1e6).view(np.int32))          # bit patterns of eps
    bound = lambda bits: np.isfinite(gn.groupnorm_act(gn.NONE, x, 2, gamma, beta, float(np.int32(bits).view(np.float32)))[1][0, 0, 0])
    assert bound(hi) and not bound(lo)
    while hi - lo > 1:
        mid = (lo + hi) // 2
        lo, hi = (lo, mid) if bound(mid) else (mid, hi)
    eps = float(np.int32(hi + 2).view(np.float32))
    y, tau = tao.tao_bound_groupnorm_act(*cuda(x), 2, *cuda(gamma, beta), eps, act=kinds(tao)[act])
    ye, te, E = gn.groupnorm_act(act, x, 2, gamma, beta, eps)
    assert_outputs(y[..., 5:], tau[..., 5:], ye[..., 5:], te[..., 5:], E[..., 5:], act)
    assert (tau[..., :5].cpu().numpy() >= te[..., :5] * (1 - np.longdouble(2) ** -58)).all()
