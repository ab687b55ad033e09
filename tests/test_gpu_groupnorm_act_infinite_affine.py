"""Infinite gammas and betas of the GroupNorm with an activation: no bound (NaN) for their channel, so that no claim is admitted there."""
import numpy as np
import pytest
import torch

import oracle
from oracle import groupnorm_act as gn
from opmap import assert_profile_equal


def inputs(B, P, C, seed):
    rng = np.random.default_rng(seed)
    x = rng.normal(0, 1, (B, P, C)).astype(np.float32)
    gamma, beta = rng.normal(1, 0.3, C).astype(np.float32), rng.normal(0, 0.5, C).astype(np.float32)
    gamma[1], gamma[C - 2], beta[3], beta[C - 1] = np.inf, -np.inf, np.inf, -np.inf
    return x, gamma, beta, ~(np.isfinite(gamma) & np.isfinite(beta))


@pytest.mark.parametrize("act", [gn.NONE, gn.RELU, gn.SILU])
def test_the_oracle_has_no_bound_there(act):
    x, gamma, beta, none = inputs(2, 5, 12, 1)
    tau = gn.groupnorm_act(act, x, 3, gamma, beta)[1]
    assert np.isnan(tau[..., none]).all() and not np.isnan(tau[..., ~none]).any()


@pytest.fixture(scope="module")
def tao():
    import paper_2510_16028_amd as t
    return t


# (groups of a workgroup each, and larger ones; channels in fours, twos and ones)
@pytest.mark.gpu
@pytest.mark.parametrize("B,P,C,groups", [(2, 20, 24, 4), (2, 20, 26, 2), (1, 31, 35, 5), (1, 5000, 8, 2), (1, 6000, 10, 2), (1, 9000, 7, 1), (2, 900, 520, 4)])
@pytest.mark.parametrize("act", [gn.NONE, gn.RELU, gn.SILU])
def test_infinite_gammas_and_betas(tao, B, P, C, groups, act):
    kind = {gn.NONE: tao.ACT_EXACT, gn.RELU: tao.ACT_RELU, gn.SILU: tao.ACT_SILU}[act]
    x, gamma, beta, none = inputs(B, P, C, P + C)
    xd, gd, bd = (torch.from_numpy(a).cuda() for a in (x, gamma, beta))
    y, tau = tao.tao_bound_groupnorm_act(xd, groups, gd, bd, act=kind)
    nd = torch.from_numpy(none).cuda()
    assert bool(torch.isnan(tau[..., nd]).all()) and bool(torch.isfinite(tau[..., ~nd]).all())
    # the other channels are those of finite gammas and betas, bit for bit
    y0, tau0 = tao.tao_bound_groupnorm_act(xd, groups, torch.where(nd, 1.0, gd), torch.where(nd, 0.0, bd), act=kind)
    assert torch.equal(y[..., ~nd], y0[..., ~nd]) and torch.equal(tau[..., ~nd], tau0[..., ~nd])
    for claimed, y_ref in ((torch.where(nd, 5.0, y), None), (torch.where(nd, 5.0, y), torch.where(nd, 7.0, y)), (torch.where(nd, 7.0, y), torch.where(nd, 7.0, y))):
        pf = tao.tao_bound_check_groupnorm_act(xd, claimed, groups, gd, bd, act=kind, y_ref=y_ref)
        other = y if y_ref is None else y_ref
        assert_profile_equal(pf, oracle.check_and_profile(claimed.cpu().numpy(), other.cpu().numpy(), tau.cpu().numpy()))
        assert pf["violations"] == B * P * none.sum()
