"""The check of an 8-bit product whose batch is padded with rows of zeros: outputs and bounds of 0, which admit a claim of 0 and nothing else, and cost no more than
other elements."""
import pytest
import torch

import oracle
from opmap import assert_profile_equal

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tao():
    import paper_2510_16028_amd as t
    return t


def padded(tao, M, N, K, share, with_bias=False):
    g = torch.Generator(device="cuda").manual_seed(M + N)
    A, W = (torch.randint(-127, 128, (n, K), generator=g, device="cuda", dtype=torch.int8) for n in (M, N))
    sa, sw = (torch.rand(n, generator=g, device="cuda") * 0.01 + 0.01 for n in (M, N))
    rows = torch.arange(M, device="cuda") >= int(M * (1 - share))
    A[rows] = 0
    sa[rows] = 0
    return g, (A, sa, W, sw), torch.randn(N, generator=g, device="cuda") if with_bias else None, rows


@pytest.mark.parametrize("M,N,K", [(5, 100, 70), (60, 301, 96), (300, 260, 512), (1500, 1800, 64), (2100, 2100, 64)])
@pytest.mark.parametrize("with_bias", [False, True])
@pytest.mark.parametrize("ref", [False, True])
def test_padded_rows(tao, M, N, K, with_bias, ref):
    g, a, bias, rows = padded(tao, M, N, K, 0.5, with_bias)
    y, tau = tao.tao_bound_linear_int8(*a, bias=bias)
    if not with_bias:
        assert bool((y[rows] == 0).all()) and bool((tau[rows] == 0).all())
    y_ref = y.clone() if ref else None
    check = lambda c: tao.tao_bound_check_linear_int8(*a, c, bias=bias, y_ref=y_ref)
    reference = lambda c: oracle.check_and_profile(c.cpu().numpy(), y.cpu().numpy(), tau.cpu().numpy())
    assert check(y.clone())["accept"] == 1
    first = int(torch.nonzero(rows)[0])
    for v in (-0.0, 1e-45, -1e-38, 2.0 ** -91, 1.0, float("nan"), float("-inf")):
        claimed = y.clone()
        claimed[first:, ::7] = v
        pf = check(claimed)
        assert_profile_equal(pf, reference(claimed), str(v))
        if not with_bias:
            assert pf["violations"] == (0 if v == 0 else claimed[first:, ::7].numel()), v


@pytest.mark.parametrize("v", [float("inf"), float("nan"), 3e38])
def test_claims_equal_to_given_outputs_that_are_no_ordinary_numbers(tao, v):
    _, a, _, _ = padded(tao, 40, 64, 96, 0.25)
    y, tau = tao.tao_bound_linear_int8(*a)
    y[3, 8:20] = v
    pf = tao.tao_bound_check_linear_int8(*a, y.clone(), y_ref=y)
    assert_profile_equal(pf, oracle.check_and_profile(y.cpu().numpy(), y.cpu().numpy(), tau.cpu().numpy()))
    assert pf["violations"] == (0 if v == 3e38 else 12)


def test_what_padding_costs(tao):
    """Half of the rows padded against none, claims equal to their outputs, in turn: 1.0 times as long as measured, 1.45 where zeros are checked one by one."""
    M, N, K = 2048, 8192, 1024
    out, ws = tao.new_profile_buffer(torch.device("cuda", 0)), torch.empty(tao.tao_check_workspace_bytes(M * N), dtype=torch.uint8, device="cuda")
    calls = []
    for share in (0.0, 0.5):
        _, a, _, _ = padded(tao, M, N, K, share)
        y, _ = tao.tao_bound_linear_int8(*a)
        calls.append(lambda a=a, y=y: tao.tao_bound_check_linear_int8(*a, y, out=out, ws=ws, readback=False))
    best = [float("inf")] * 2
    e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    for _ in range(8):
        for i, f in enumerate(calls):
            f()
            e0.record()
            for _ in range(10):
                f()
            e1.record()
            e1.synchronize()
            best[i] = min(best[i], e0.elapsed_time(e1))
    assert best[1] < 1.25 * best[0], best
