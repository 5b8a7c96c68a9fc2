"""The polynomial that stands in for a part of the exponentials, evaluated as the kernels do (32 bits, fused multiply-adds)."""
import os
import re

import numpy as np

SOURCE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2407_14057_b200", "csrc",
                      "attn_common.cuh")


def coefficients():
    """Highest power first, as they stand in the source."""
    text = open(SOURCE).read()
    body = text[text.index("ex2_poly_x2("):]
    return [float.fromhex(c) for c in re.findall(r"f32x2_pack\((0x[0-9a-fp.+-]+?)f, \1f\)", body[:body.index("\n}\n")])]


def exp2_poly(x):
    """x float32 -> 2^x as the kernel has it."""
    x = np.maximum(x.astype(np.float32), np.float32(-126.0))   # numpy keeps NaN, as max.NaN does
    n = np.rint(x)
    f = x.astype(np.float64) - n
    c = coefficients()
    p = np.full(x.shape, c[0])
    for a in c[1:]:   # the product of two 24-bit numbers is exact in 64 bits: one rounding, to 32
        p = (p * f + a).astype(np.float32).astype(np.float64)
    return (p * np.exp2(n)).astype(np.float32)


def test_coefficients_are_six_numbers_of_32_bits():
    c = coefficients()
    assert len(c) == 6 and all(float(np.float32(a)) == a for a in c)


def test_error_over_one_period():
    """Within 1.6e-7 of itself (2.7 half steps of a 24-bit number), on average within 3e-8 of zero: a sum is not lifted."""
    x = np.linspace(-0.5, 0.5, 400001).astype(np.float32)
    e = exp2_poly(x).astype(np.float64) / np.exp2(x.astype(np.float64)) - 1.0
    assert np.abs(e).max() < 1.6e-7 and abs(e.mean()) < 3e-8


def test_whole_powers_are_exact():
    n = np.arange(-126, 127, dtype=np.float32)
    assert np.array_equal(exp2_poly(n), np.exp2(n))


def test_error_over_the_range_and_below_it():
    x = np.random.default_rng(0).uniform(-126, 126, 400000).astype(np.float32)
    e = exp2_poly(x).astype(np.float64) / np.exp2(x.astype(np.float64)) - 1.0
    assert np.abs(e).max() < 1.6e-7
    assert np.array_equal(exp2_poly(np.array([-127.0, -1e30, -np.inf])), np.full(3, 2.0 ** -126, np.float32))
    assert np.isnan(exp2_poly(np.array([np.nan]))[0])
