"""Infinite scales and biases of the 8-bit product: no bound (NaN), so that no claim of such a row or column is admitted, finite ones least of all."""
import numpy as np
import pytest
import torch

import oracle
from oracle import int8
from opmap import assert_profile_equal

INF = float("inf")


def operands(M, N, K, seed):
    rng = np.random.default_rng(seed)
    A, W = rng.integers(-128, 128, (M, K), dtype=np.int8), rng.integers(-128, 128, (N, K), dtype=np.int8)
    sa, sw, b = rng.uniform(0.001, 0.1, M).astype(np.float32), rng.uniform(0.001, 0.1, N).astype(np.float32), rng.normal(0, 1, N).astype(np.float32)
    sa[1], sw[6], b[9], b[14] = np.inf, -np.inf, np.inf, -np.inf
    if K:
        A[2], W[7] = 0, 0
    none = ~(np.isfinite(sa)[:, None] & np.isfinite(sw)[None, :] & np.isfinite(b)[None, :])
    return A, sa, W, sw, b, none


class Model:
    u, mode, lam, flags = 2.0 ** -24, 0, 4.0, 1


@pytest.mark.parametrize("model", [None, Model])
@pytest.mark.parametrize("K", [0, 1, 40])
def test_the_oracle_has_no_bound_there(K, model):
    A, sa, W, sw, b, none = operands(5, 21, K, K)
    for bias in (b, None):
        gone = none if bias is not None else ~(np.isfinite(sa)[:, None] & np.isfinite(sw)[None, :])
        assert np.array_equal(np.isnan(int8.linear_int8(A, sa, W, sw, bias, model=model)[1]), gone)


@pytest.fixture(scope="module")
def tao():
    import paper_2510_16028_amd as t
    return t


@pytest.mark.gpu
@pytest.mark.parametrize("flags", [0, 1])
@pytest.mark.parametrize("M,N,K", [(4, 40, 64), (3, 33, 0), (70, 90, 200), (300, 260, 1024), (1500, 1800, 64)])
def test_infinite_operands(tao, M, N, K, flags):
    A, sa, W, sw, b, none = operands(M, N, K, M + K)
    d = [torch.from_numpy(np.ascontiguousarray(a)).cuda() for a in (A, sa, W, sw, b)]
    model = tao.FpModel(flags=flags)
    for bias in (d[4], None):
        gone = none if bias is not None else ~(np.isfinite(sa)[:, None] & np.isfinite(sw)[None, :])
        y, tau = tao.tao_bound_linear_int8(*d[:4], bias=bias, model=model)
        t = tau.cpu().numpy()
        assert np.array_equal(np.isnan(t), gone)
        ordinary = torch.from_numpy(~gone).cuda()
        for claimed, y_ref in ((torch.where(ordinary, y, 5.0), None), (torch.where(ordinary, y, 5.0), torch.where(ordinary, y, 7.0)), (y.clone(), None)):
            pf = tao.tao_bound_check_linear_int8(*d[:4], claimed, bias=bias, y_ref=y_ref, model=model)
            other = y if y_ref is None else y_ref
            assert_profile_equal(pf, oracle.check_and_profile(claimed.cpu().numpy(), other.cpu().numpy(), t))
            assert pf["violations"] == gone.sum()


@pytest.mark.gpu
def test_finite_operands_beyond_the_binary32_range_have_an_infinite_bound(tao):
    """The bound of 16384 (3e38)^2 is beyond the range, and is said to be; no operand is infinite."""
    one = torch.ones(1, device="cuda")
    A = torch.full((1, 128), 127, dtype=torch.int8, device="cuda")
    y, tau = tao.tao_bound_linear_int8(A, 3e38 * one, A, 3e38 * one)
    assert float(y) == float(tau) == INF
