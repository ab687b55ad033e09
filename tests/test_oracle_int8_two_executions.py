"""Two honest executions of the 8-bit product, checked against each other: within 2 tau always, and not within tau."""
import numpy as np
import pytest

import oracle
from oracle import int8


@pytest.mark.parametrize("with_bias", [False, True])
@pytest.mark.parametrize("K", [64, 3000])
def test_alpha_2_admits_every_order_of_the_scales_and_alpha_1_only_its_own(with_bias, K):
    rng = np.random.default_rng(K)
    f = np.float32
    A, W = rng.integers(-127, 128, (300, K), dtype=np.int8), rng.integers(-127, 128, (400, K), dtype=np.int8)
    sa, sw = rng.uniform(0.01, 0.04, 300).astype(f), rng.uniform(0.0005, 0.001, 400).astype(f)
    b = rng.normal(0, 0.5, 400).astype(f) if with_bias else None
    y, tau = int8.linear_int8(A, sa, W, sw, b)
    tau = tau.astype(f)
    tau = np.where(tau.astype(np.longdouble) < int8.linear_int8(A, sa, W, sw, b)[1], np.nextafter(tau, f(np.inf)), tau)
    S = (A.astype(np.int64) @ W.astype(np.int64).T).astype(f)
    end = lambda v: v if b is None else v + b
    orders = [end((S * sa[:, None]) * sw), end((S * sw) * sa[:, None]), end(S * (sa[:, None] * sw))]
    if b is not None:                                        # the last two steps fused: one rounding (binary64 holds the product)
        orders.append(((S * sa[:, None]).astype(np.float64) * sw + b).astype(f))
    for i, claimed in enumerate(orders):
        assert oracle.check_and_profile(claimed, y, tau, 2.0)["violations"] == 0
        outside = oracle.check_and_profile(claimed, y, tau, 1.0)["violations"]
        if i == 0:
            assert outside == 0
        elif i < 3:
            assert 0.001 * y.size < outside < 0.01 * y.size
