"""How far the quantisation of rows, whose scale is the product with fl(1/127), lies from that of a program that divides by 127: one step of the scale in one
row of twenty, and one step of values next to the middle of two whole numbers."""
import numpy as np

from oracle import int8

f = np.float32


def test_scales_are_the_quotients_or_a_step_below():
    """All leading digits; the exponent moves both alike."""
    m = (np.arange(1 << 23, dtype=np.uint32) | np.uint32(0x3f800000)).view(f)
    product, quotient = m * (f(1) / f(127)), m / f(127)
    step = quotient.view(np.int32) - product.view(np.int32)
    assert set(np.unique(step)) == {0, 1}
    assert 0.046 < (step == 1).mean() < 0.048
    some = np.arange(0, 1 << 23, 8191)
    assert np.array_equal(int8.quantize_rows(m[some, None])[1], product[some])


def test_values_differ_next_to_the_middle_of_two_alone():
    rng = np.random.default_rng(3)
    x = (rng.normal(0, 1, (4000, 512)) * np.exp(rng.normal(0, 3, (4000, 1)))).astype(f)
    # arguments in the middle of two, which a step of the scale moves to either side
    s = np.abs(x).max(axis=1) / f(127)
    x[:, 1:255] = np.where(np.abs((np.arange(-127, 127) + f(0.5)) * s[:, None]) < np.abs(x).max(axis=1, keepdims=True), (np.arange(-127, 127) + f(0.5)) * s[:, None], x[:, 1:255])
    q, scale = int8.quantize_rows(x)
    other = np.abs(x).max(axis=1) / f(127)
    q2 = np.clip(np.rint(x / other[:, None]), -127, 127).astype(np.int8)
    same_scale = scale == other
    assert np.array_equal(q[same_scale], q2[same_scale])
    apart = q != q2
    assert apart.any() and (np.abs(q.astype(int) - q2) <= 1).all()
    # a step of the scale is at most 2^-23 of it, either quotient's rounding half a step: 127 (2^-23 + 2 2^-24) of a whole number at most
    ratio = np.abs(x.astype(np.float64) / other[:, None].astype(np.float64))
    assert (np.abs(ratio - np.floor(ratio) - 0.5)[apart] <= 127 * 2.0 ** -22).all()
