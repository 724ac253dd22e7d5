"""The gated quantizer where exp(-g) leaves the middle of fp32's range, against the definition in 64 bits.

Tolerance, derived before the first run: h = g / (1 + exp(-g)) * u in fp32.  2^x from the special function unit is within 2
ulp (2.4e-7), what the split of the exponent leaves out within 1e-7 at |g| = 90 (the square of 90 * 4.9e-6, halved), and four
roundings follow (2.4e-7): h is within 6e-7 of its value, and a code differs only where h / scale is that near a rounding
boundary.  exp(-g) above fp32's largest number is infinite (g < -88.73): h is zero there, by the formula in fp32."""
import numpy as np
import pytest

from .test_gpu_fp8 import plain_quantize, plain_quantize_with, st  # noqa: F401

pytestmark = pytest.mark.gpu

FLT_MAX = 3.4028234663852886e38


def definition(v, F):
    g, u = v[:, :F], v[:, F:]
    with np.errstate(over="ignore"):
        e = np.exp(-g)
        return g / (1.0 + np.where(e > FLT_MAX, np.inf, e)) * u


def holds(st, x):
    F = x.shape[1] // 2
    codes, scale = st.stamp_fp8_gated_quantize(x)
    h = definition(x.double().cpu().numpy(), F)
    c, s = plain_quantize(h)
    got = codes.double().cpu().numpy()
    assert np.array_equal(scale.double().cpu().numpy(), s)
    lo, hi = plain_quantize_with(h * (1 - 6e-7), s), plain_quantize_with(h * (1 + 6e-7), s)
    assert np.all((got == c) | (got == lo) | (got == hi))
    return got


# (-88.7 rounds to -88.5 in bf16)
@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("u", [1.0, -1.25 * 2.0 ** 20, 1.7 * 2.0 ** 100])
@pytest.mark.parametrize("g", [-79.5, -80.5, -86.0, -87.0, -87.5, -88.0, -88.5, -88.7, -89.0, -90.5, -200.0])
def test_blocks_of_gates_far_below_zero(st, g, u, dtype):
    import torch
    F = 256
    x = torch.empty(3, 2 * F, device="cuda")
    x[:, :F], x[:, F:] = g, u
    x[1, F:] *= torch.linspace(0.5, 1.0, F, device="cuda")     # one gate, ups of many sizes
    x[2, 128:F] = -3.0                                         # a block of such gates beside an ordinary one
    got = holds(st, x.to(getattr(torch, dtype)))
    if g >= -88.7:
        assert np.all(got[0] != 0)


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
def test_gates_of_every_size_in_one_block(st, dtype):
    import torch
    g = torch.Generator(device="cuda").manual_seed(5)
    F, M = 640, 200
    x = torch.empty(M, 2 * F, device="cuda")
    x[:, :F] = torch.rand(M, F, generator=g, device="cuda") * 180 - 88.7
    x[:, F:] = torch.randn(M, F, generator=g, device="cuda")
    x[: M // 2, :F] = -x[: M // 2, :F].abs().clamp_max_(88.7)  # below zero only: h spans what fp32 does
    x[::7, :F] *= 1e-3
    x[3, :F] = torch.linspace(1e30, 8e37, F, device="cuda")    # large gates: h is g u
    x[3, F:] = 0.5
    holds(st, x.to(getattr(torch, dtype)))
