"""The product with an epilogue refuses bad arguments on the host, before anything is launched (no GPU needed)."""
import ctypes

import pytest

from .test_fp8_abi import A, B, BF16, F32, INVALID, ODD, OK, UNSUPPORTED, p, st  # noqa: F401

R = 1 << 30   # an address far from the others


def fused(st, x=A, xs=A, w=A, ws=A, bias=0, act=0, residual=0, r_dtype=BF16, ldr=64, M=4, N=64, K=256, Y=B, dtype=BF16):  # noqa: F811
    return st.lib().stamp_fp8_linear_fused(p(x), p(xs), p(w), p(ws), p(bias), act, p(residual), r_dtype, ctypes.c_longlong(ldr), M, N, K, p(Y), dtype, p(0))


def quantized(st, x=A, xs=A, w=A, ws=A, bias=0, act=0, M=4, N=64, K=256, codes=B, scale=B):  # noqa: F811
    return st.lib().stamp_fp8_linear_quantized(p(x), p(xs), p(w), p(ws), p(bias), act, M, N, K, p(codes), p(scale), p(0))


@pytest.mark.parametrize("call,bad", [
    (fused, dict(x=0)), (fused, dict(xs=0)), (fused, dict(w=0)), (fused, dict(ws=0)), (fused, dict(Y=0)), (fused, dict(M=-1)), (fused, dict(N=0)),
    (fused, dict(dtype=2)), (fused, dict(act=-1)), (fused, dict(act=5)), (fused, dict(x=ODD)), (fused, dict(Y=B + 1)),
    (fused, dict(residual=R, r_dtype=2)), (fused, dict(residual=R, ldr=63)), (fused, dict(residual=R + 1)), (fused, dict(residual=R + 2, r_dtype=F32)),
    (fused, dict(residual=B, ldr=65)), (fused, dict(residual=B + 2)), (fused, dict(residual=B, r_dtype=F32)),
    (fused, dict(residual=B - 64 * 8 + 2)), (fused, dict(residual=B + 4 * 64 * 2 - 2)),
    (fused, dict(residual=B, r_dtype=F32, dtype=F32, act=1, K=4112)),
    (quantized, dict(x=0)), (quantized, dict(codes=0)), (quantized, dict(scale=0)), (quantized, dict(codes=ODD)), (quantized, dict(act=9)), (quantized, dict(K=0)),
    (quantized, dict(N=256, codes=A)), (quantized, dict(codes=A + 4 * 256 - 16)), (quantized, dict(codes=A - 4 * 64 + 16)),
])
def test_invalid_arguments(st, call, bad):  # noqa: F811
    assert call(st, **bad) == INVALID
    assert st.stamp_last_launch_count() == 0


@pytest.mark.parametrize("call,bad", [
    (fused, dict(K=100)), (fused, dict(M=(1 << 30) + 1)), (fused, dict(K=(1 << 31) - 16)), (fused, dict(residual=R, ldr=1 << 60)),
    (quantized, dict(N=40)), (quantized, dict(K=8)), (quantized, dict(M=(1 << 30) + 1)),
])
def test_unsupported_sizes(st, call, bad):  # noqa: F811
    assert call(st, **bad) == UNSUPPORTED
    assert st.stamp_last_launch_count() == 0


def test_zero_rows_need_no_buffers_and_launch_nothing(st):  # noqa: F811
    assert fused(st, M=0, x=0, xs=0, Y=0) == OK
    assert fused(st, M=0, x=0, xs=0, Y=0, residual=R) == OK
    assert quantized(st, M=0, x=0, xs=0, codes=0, scale=0) == OK
    assert st.stamp_last_launch_count() == 0


def test_the_marshalling_module_refuses_what_is_not_a_cuda_tensor(st):  # noqa: F811
    import torch
    c, s = torch.zeros(4, 256).to(torch.float8_e4m3fn), torch.zeros(4, 2, dtype=torch.uint8).view(torch.float8_e8m0fnu)
    for bad in (lambda: st.stamp_fp8_linear_fused(c, s, c, s), lambda: st.stamp_fp8_linear_fused(c, s, None, s), lambda: st.stamp_fp8_linear_quantized(c, s, c, s),
                lambda: st.stamp_fp8_linear_quantized(1, s, c, s), lambda: st.calls().fp8_linear_fused(c), lambda: st.calls().fp8_linear_quantized(c)):
        with pytest.raises(ValueError):
            bad()


FAR = 1 << 40


# Another CTA may still read what one writes: an output shares no memory with an input, but for a residual updated in place.
@pytest.mark.parametrize("call,bad", [
    (fused, dict(x=FAR, Y=FAR)), (fused, dict(x=FAR, Y=FAR + 4 * 256 - 16)), (fused, dict(x=FAR + 4 * 64 * 2 - 16, Y=FAR)),
    (fused, dict(xs=FAR, Y=FAR)), (fused, dict(xs=FAR + 4 * 64 * 2 - 1, Y=FAR)), (fused, dict(xs=FAR - 7, Y=FAR)),
    (fused, dict(w=FAR, Y=FAR)), (fused, dict(ws=FAR + 2, Y=FAR)), (fused, dict(bias=FAR + 8, Y=FAR)),
    (quantized, dict(xs=FAR, scale=FAR)), (quantized, dict(xs=FAR + 3, scale=FAR)), (quantized, dict(xs=FAR - 7, scale=FAR)), (quantized, dict(xs=FAR, codes=FAR)),
    (quantized, dict(x=FAR, scale=FAR + 4 * 256 - 1)), (quantized, dict(codes=FAR, scale=FAR + 4 * 64 - 1)), (quantized, dict(codes=FAR, scale=FAR - 3)),
    (quantized, dict(w=FAR, codes=FAR, scale=R)), (quantized, dict(ws=FAR, codes=FAR, scale=R)), (quantized, dict(bias=FAR, codes=FAR, scale=R)), (quantized, dict(w=FAR, scale=FAR)),
])
def test_outputs_over_inputs_are_refused(st, call, bad):  # noqa: F811
    assert call(st, **{**(dict(codes=2 * FAR, scale=R) if call is quantized else {}), **bad}) == INVALID
    assert st.stamp_last_launch_count() == 0
