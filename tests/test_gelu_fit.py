"""The fit behind the fused product's GELU, as its coefficients stand in the kernel's source, against the scaled complementary
error function: Phi(-x) = exp(-x^2 / 2) R(x), R(x) = erfcx(x / sqrt 2) / 2 = t P(1 - 2 t), t = 1 / (1 + x / 3)  (no GPU needed)."""
import os
import re

import numpy as np

SOURCE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2510_26771_b200", "csrc", "k_fp8_gemm.cuh")


def coefficients():
    with open(SOURCE) as f:
        found = re.search(r"constexpr float P\[9\] = \{([^}]*)\}", f.read())
    p = [np.float32(c.rstrip("f")) for c in found.group(1).split(", ")]
    assert len(p) == 9
    return p


def error(x, dtype):
    from scipy.special import erfcx
    want = 0.5 * erfcx(x / np.sqrt(2.0))
    x = x.astype(dtype)
    t = dtype(1) / (dtype(1) + x * dtype(np.float32(1 / 3)) if dtype is np.float32 else 1 + x / 3)
    u = dtype(1) - dtype(2) * t
    r = np.zeros_like(x)
    for c in reversed(coefficients()):
        r = r * u + dtype(c)
    return np.max(np.abs(r.astype(np.float64) * t - want) / want)


def test_the_fit_is_within_the_error_that_its_comment_states():
    """2^-23.3 up to 14, where exp(-x^2 / 2) vanishes from fp32; scipy's erfcx is good to some 2^-50."""
    assert error(np.linspace(0.0, 14.0, 200001), np.float64) <= 2.0 ** -23.3


def test_the_fit_in_fp32():
    """Nine roundings of a sum whose terms fall off quickly, and the reciprocal's: R within 2^-21."""
    assert error(np.linspace(0.0, 14.0, 200001).astype(np.float32).astype(np.float64), np.float32) <= 2.0 ** -21
