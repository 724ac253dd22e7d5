"""The block-scaled 8-bit floating point calls refuse bad arguments on the host, before anything is launched (no GPU needed):
through the C ABI by status, through the marshalling module by exception."""
import ctypes

import pytest

from paper_2510_26771_b200 import build as stamp_build

F32, BF16 = 0, 1
OK, INVALID, UNSUPPORTED = 0, 1, 2


@pytest.fixture(scope="module")
def st():
    stamp_build.build()
    from paper_2510_26771_b200 import binding
    binding.lib()
    return binding


def p(address):
    return ctypes.c_void_p(address)


A, B, ODD = 4096, 8192, 4100   # never dereferenced: the checks below fail first


def quantize(st, X=A, dtype=BF16, ldx=256, rows=0, T=4, M=4, K=256, codes=B, scale=B):
    return st.lib().stamp_fp8_quantize(p(X), dtype, ctypes.c_longlong(ldx), p(rows), T, M, K, p(codes), p(scale), p(0))


def gated(st, X=A, dtype=BF16, ldx=512, M=4, F=256, codes=B, scale=B):
    return st.lib().stamp_fp8_gated_quantize(p(X), dtype, ctypes.c_longlong(ldx), M, F, p(codes), p(scale), p(0))


def weights(st, W=A, dtype=BF16, E=1, N=64, K=256, codes=B, scale=B):
    return st.lib().stamp_fp8_quantize_weights(p(W), dtype, E, N, K, p(codes), p(scale), p(0))


def linear(st, x=A, xs=A, w=A, ws=A, bias=0, M=4, N=64, K=256, Y=B, dtype=BF16):
    return st.lib().stamp_fp8_linear(p(x), p(xs), p(w), p(ws), p(bias), M, N, K, p(Y), dtype, p(0))


def grouped(st, x=A, xs=A, offsets=A, w=A, ws=A, bias=0, M=4, E=3, N=64, K=256, Y=B, dtype=BF16):
    return st.lib().stamp_fp8_linear_grouped(p(x), p(xs), p(offsets), p(w), p(ws), p(bias), M, E, N, K, p(Y), dtype, p(0))


@pytest.mark.parametrize("call,bad", [
    (quantize, dict(X=0)), (quantize, dict(codes=0)), (quantize, dict(scale=0)), (quantize, dict(X=ODD)), (quantize, dict(codes=ODD)),
    (quantize, dict(dtype=2)), (quantize, dict(M=-1)), (quantize, dict(T=-1)), (quantize, dict(K=0)), (quantize, dict(ldx=255)),
    (quantize, dict(ldx=260)), (quantize, dict(M=5)), (quantize, dict(dtype=F32, ldx=257)),
    (gated, dict(X=0)), (gated, dict(ldx=511)), (gated, dict(F=0)), (gated, dict(dtype=-1)), (gated, dict(scale=0)), (gated, dict(M=-2)),
    (weights, dict(W=0)), (weights, dict(E=0)), (weights, dict(N=0)), (weights, dict(dtype=7)), (weights, dict(W=ODD)),
    (linear, dict(x=0)), (linear, dict(xs=0)), (linear, dict(w=0)), (linear, dict(ws=0)), (linear, dict(Y=0)), (linear, dict(M=-1)),
    (linear, dict(N=0)), (linear, dict(K=0)), (linear, dict(dtype=3)), (linear, dict(x=ODD)), (linear, dict(w=ODD)), (linear, dict(Y=B + 1)),
    (linear, dict(Y=B + 2, dtype=F32)),
    (grouped, dict(offsets=0)), (grouped, dict(E=0)), (grouped, dict(w=0)), (grouped, dict(M=-1)), (grouped, dict(Y=0)),
])
def test_invalid_arguments(st, call, bad):
    assert call(st, **bad) == INVALID
    assert st.stamp_last_launch_count() == 0


@pytest.mark.parametrize("call,bad", [
    (quantize, dict(K=250, ldx=256)), (quantize, dict(K=8, ldx=256)), (gated, dict(F=100)), (weights, dict(K=72)), (weights, dict(E=65536)),
    (linear, dict(K=100)), (linear, dict(M=(1 << 30) + 1)), (grouped, dict(E=1025)), (grouped, dict(K=24)), (grouped, dict(E=1024, N=1 << 22)),
])
def test_unsupported_sizes(st, call, bad):
    assert call(st, **bad) == UNSUPPORTED
    assert st.stamp_last_launch_count() == 0


def test_zero_rows_need_no_buffers_and_launch_nothing(st):
    assert quantize(st, M=0, X=0, codes=0, scale=0) == OK
    assert gated(st, M=0, X=0, codes=0, scale=0) == OK
    assert linear(st, M=0, x=0, xs=0, Y=0) == OK
    assert grouped(st, M=0, x=0, xs=0, Y=0) == OK
    assert st.stamp_last_launch_count() == 0


def test_the_marshalling_module_refuses_what_is_not_a_cuda_tensor(st):
    import torch
    x = torch.zeros(4, 256, dtype=torch.bfloat16)
    c, s = torch.zeros(4, 256).to(torch.float8_e4m3fn), torch.zeros(4, 2, dtype=torch.uint8).view(torch.float8_e8m0fnu)
    for bad in (lambda: st.stamp_fp8_quantize(x), lambda: st.stamp_fp8_quantize(None), lambda: st.stamp_fp8_gated_quantize(x),
                lambda: st.stamp_fp8_gated_quantize([1, 2]), lambda: st.stamp_fp8_linear(c, s, c, s), lambda: st.stamp_fp8_linear(c, s, None, s),
                lambda: st.stamp_fp8_linear_grouped(c, s, None, c, s), lambda: st.calls().fp8_quantize(x),
                lambda: st.stamp_fp8_quantize_weights(x)):
        with pytest.raises(ValueError):
            bad()
