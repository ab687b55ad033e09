"""The check of a GroupNorm with ReLU: most elements below 0 have an output and a bound of 0, which admits a claim of 0 and nothing else, and costs no more than
any other element."""
import pytest
import torch

import oracle
from opmap import assert_profile_equal

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tao():
    import paper_2510_16028_amd as t
    return t


@pytest.mark.parametrize("B,P,C,groups", [(2, 64, 320, 32), (1, 3000, 64, 8), (1, 1500, 35, 5), (3, 40, 6, 2)])
@pytest.mark.parametrize("ref", [False, True])
def test_a_bound_of_0_admits_0_alone(tao, B, P, C, groups, ref):
    g = torch.Generator(device="cuda").manual_seed(P)
    x = torch.randn((B, P, C), generator=g, device="cuda")
    y, tau = tao.tao_bound_groupnorm_act(x, groups, act=tao.ACT_RELU)
    none = (tau == 0) & (y == 0)
    assert none.float().mean() > 0.4
    y_ref = y.clone() if ref else None
    check = lambda c: tao.tao_bound_check_groupnorm_act(x, c, groups, act=tao.ACT_RELU, y_ref=y_ref)
    reference = lambda c: oracle.check_and_profile(c.cpu().numpy(), y.cpu().numpy(), tau.cpu().numpy())
    places = torch.nonzero(none.flatten()).flatten()
    places = places[torch.randperm(len(places), generator=g, device="cuda")[:37]]
    for v in (-0.0, 1e-45, -1e-45, 1e-38, 2.0 ** -91, -2.0 ** -89, 1e-20, 1.0, float("nan"), float("inf")):
        claimed = y.clone()
        claimed.view(-1)[places] = v
        pf = check(claimed)
        assert_profile_equal(pf, reference(claimed), str(v))
        assert pf["violations"] == (0 if v == 0 else len(places)), v
    assert_profile_equal(check(-y), reference(-y))


def test_what_it_costs(tao):
    """Next to the check without an activation, of as much traffic, in turn: 1.08 times as long as measured, 1.5 where bounds of 0 are checked one by one."""
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn((4, 16384, 512), generator=g, device="cuda")
    ws = torch.empty(tao.tao_bound_check_groupnorm_act_workspace_bytes(4, 16384, 512, 32), dtype=torch.uint8, device="cuda")
    out = tao.new_profile_buffer(x.device)
    calls = []
    for act in (tao.ACT_EXACT, tao.ACT_RELU):
        y, _ = tao.tao_bound_groupnorm_act(x, 32, act=act)
        y = torch.where(y.abs() > 1e-30, (y.view(torch.int32) + torch.randint(-1, 2, y.shape, generator=g, device="cuda", dtype=torch.int32)).view(torch.float32), y)
        calls.append(lambda act=act, y=y: tao.tao_bound_check_groupnorm_act(x, y, 32, act=act, out=out, ws=ws, readback=False))
    best = [float("inf")] * 2
    a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    for _ in range(8):
        for i, f in enumerate(calls):
            f()
            a.record()
            for _ in range(10):
                f()
            b.record()
            b.synchronize()
            best[i] = min(best[i], a.elapsed_time(b))
    assert best[1] < 1.3 * best[0], best
