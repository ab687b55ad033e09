"""The SiLU bound where the slope of the activation vanishes, in small groups, whose bounds are small: far out on the negative side, and about the
slope's zero at -1.278."""
import numpy as np
import pytest
import torch

from oracle import groupnorm_act as gn

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tao():
    import paper_2510_16028_amd as t
    return t


# (gamma and beta: where the arguments lie)
@pytest.mark.parametrize("per,P,B", [(2, 1, 40), (4, 1, 40), (4, 16, 4), (16, 1, 40), (3, 5, 8), (4, 5000, 1), (1, 9000, 1)])
@pytest.mark.parametrize("gamma,beta", [(20.0, 0.0), (20.0, -15.0), (60.0, -40.0), (300.0, 0.0), (1.0, -1.278), (1e-2, -1.278), (1e-4, -1.2784645), (0.5, 10.0), (0.0, -1.2784645), (1e-3, -30.0)])
def test_silu_bound_is_within_1e_6(tao, per, P, B, gamma, beta):
    rng = np.random.default_rng(per * P)
    C = 16 * per if P < 100 else 2 * per
    x = rng.normal(0.1, 1, (B, P, C)).astype(np.float32)
    g, b = (gamma * rng.uniform(0.9, 1.1, C)).astype(np.float32), (beta + 1e-3 * gamma * rng.normal(0, 1, C)).astype(np.float32)
    y, tau = tao.tao_bound_groupnorm_act(torch.from_numpy(x).cuda(), C // per, torch.from_numpy(g).cuda(), torch.from_numpy(b).cuda(), act=tao.ACT_SILU)
    te = gn.groupnorm_act(gn.SILU, x, C // per, g, b)[1]
    L = np.longdouble
    t = tau.cpu().numpy().astype(L)
    assert not np.isnan(te).any() and not np.isnan(t).any()
    # one-sided, and within 1e-6 of the formula's value; one step where it is subnormal
    assert (t >= te * (1 - L(2) ** -58)).all()
    assert (t <= te * (1 + L(1e-6)) + L(2) ** -149).all(), float((t / np.maximum(te, L(1e-300)) - 1).max())
