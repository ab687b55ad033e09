"""The check of the 8-bit product against given outputs, where single columns have no bound: the outputs are ordinary numbers there, so that only
the bound can tell, among neighbours whose claims are settled together."""
import numpy as np
import pytest
import torch

import oracle
from opmap import assert_profile_equal

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tao():
    import paper_2510_16028_amd as t
    return t


# (every tile size, and two workgroups a compute unit)
@pytest.mark.parametrize("M,N,K", [(3, 100, 70), (40, 301, 96), (300, 260, 1024), (1500, 1800, 64), (2100, 2100, 64), (4096, 4096, 32)])
@pytest.mark.parametrize("honest", [True, False])
def test_columns_without_a_bound(tao, M, N, K, honest):
    g = torch.Generator(device="cuda").manual_seed(M + N)
    r = lambda *s: torch.randn(s, generator=g, device="cuda")
    A, W = (torch.randint(-127, 128, (n, K), generator=g, device="cuda", dtype=torch.int8) for n in (M, N))
    sa, sw, bias = 0.02 + 0.01 * r(M).abs(), 0.001 + 0.001 * r(N).abs(), r(N)
    sw[5] = float("nan")
    bias[18] = float("nan")
    W[31] = 0
    sw[31] = float("inf")                                    # 0 times infinity
    sw[N - 1] = float("nan")
    none = torch.zeros(N, dtype=torch.bool, device="cuda")
    none[[5, 18, 31, N - 1]] = True
    y, tau = tao.tao_bound_linear_int8(A, sa, W, sw, bias=bias)
    assert bool(torch.isnan(tau[:, none]).all()) and bool(torch.isfinite(tau[:, ~none]).all())
    y_ref = torch.where(none, 5.0, y).contiguous()
    f = torch.tensor([0.0, 0.5, -0.5, 0.9, -3.0, 0.0, 0.2, 0.0], device="cuda")[torch.randint(0, 8, y.shape, generator=g, device="cuda")]
    claimed = y_ref if honest else torch.where(none, y_ref * (1 + 2.0 ** -20), (y_ref.double() + (f * tau).double()).float())
    for alpha in (1.0, 2.0):
        pf = tao.tao_bound_check_linear_int8(A, sa, W, sw, claimed.clone(), bias=bias, y_ref=y_ref, alpha=alpha)
        assert_profile_equal(pf, oracle.check_and_profile(claimed.cpu().numpy(), y_ref.cpu().numpy(), tau.cpu().numpy(), alpha))
        assert pf["violations"] == 4 * M if honest else pf["violations"] > 4 * M
        assert pf["accept"] == 0
