"""The bound of the 8-bit product is its formula in binary64, rounded up once."""
import numpy as np
import pytest
import torch

from oracle import int8

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tao():
    import paper_2510_16028_amd as t
    return t


# (each tile size, rows of whole units and others; sums beyond 2^24)
@pytest.mark.parametrize("M,N,K", [(1, 512, 512), (40, 301, 96), (130, 250, 1001), (300, 260, 1024), (1000, 700, 77), (20, 40, 131071)])
@pytest.mark.parametrize("with_bias", [False, True])
@pytest.mark.parametrize("model", [{}, dict(mode=1), dict(u=2.0 ** -11), dict(flags=1)])
def test_one_rounding(tao, M, N, K, with_bias, model):
    rng = np.random.default_rng(M + K)
    A, W = rng.integers(-128, 128, (M, K), dtype=np.int8), rng.integers(-128, 128, (N, K), dtype=np.int8)
    A[0], W[0] = -128, -128
    sa, sw = rng.uniform(0.001, 0.1, M).astype(np.float32), rng.uniform(-0.1, 0.1, N).astype(np.float32)
    b = rng.normal(0, 1, N).astype(np.float32) if with_bias else None
    m = tao.FpModel(**model)
    d = [None if a is None else torch.from_numpy(a).cuda() for a in (A, sa, W, sw, b)]
    tau = tao.tao_bound_linear_int8(*d[:4], bias=d[4], model=m, with_y=False)[1].cpu().numpy().astype(np.longdouble)
    te = int8.linear_int8(A, sa, W, sw, b, model=m)[1]
    L = np.longdouble
    some = te >= L(2) ** -126
    assert some.mean() > 0.98 and (tau >= te * (1 - L(2) ** -60)).all()
    # the upper rounding adds 2^-24 + 2^-32 and goes to the nearest binary32 value, half a step of 2^-23 away at most
    assert (tau[some] <= te[some] * (1 + L(2) ** -24 + L(2) ** -31) * (1 + L(2) ** -24)).all()
