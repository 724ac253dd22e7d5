"""The expert layer's calls refuse bad arguments on the host, before anything is launched (no GPU needed)."""
import ctypes

import pytest

from .test_fp8_abi import A, B, BF16, F32, INVALID, ODD, OK, UNSUPPORTED, p, st  # noqa: F401

WORKSPACE = 3
R = 1 << 30
size = ctypes.c_size_t
long_long = ctypes.c_longlong


def route(st, logits=A, dtype=F32, ldl=64, T=4, E=64, top=8, normalize=1, chosen=B, share=B, rows=B, place=B, offsets=B, row_share=B, ws=0, ws_bytes=0):  # noqa: F811
    return st.lib().stamp_expert_route(p(logits), dtype, long_long(ldl), T, E, top, normalize, p(chosen), p(share), p(rows), p(place), p(offsets), p(row_share),
                                       p(ws), size(ws_bytes), p(0))


def combine(st, y=A, dtype=F32, place=A, share=A, residual=0, r_dtype=F32, ldr=64, T=4, top=2, M=8, N=64, out=B, o_dtype=F32):  # noqa: F811
    return st.lib().stamp_expert_combine(p(y), dtype, p(place), p(share), p(residual), r_dtype, long_long(ldr), T, top, M, N, p(out), o_dtype, p(0))


def layer(st, X=A, dtype=BF16, ldx=256, rows=A, share=A, offsets=A, up=A, up_s=A, up_b=0, down=A, down_s=A, down_b=0, residual=0, r_dtype=BF16, ldr=64,  # noqa: F811
          T=4, M=8, E=3, K=256, F=128, N=64, Y=B, o_dtype=BF16, ws=A, ws_bytes=1 << 20):
    return st.lib().stamp_fp8_expert_layer(p(X), dtype, long_long(ldx), p(rows), p(share), p(offsets), p(up), p(up_s), p(up_b), p(down), p(down_s), p(down_b),
                                           p(residual), r_dtype, long_long(ldr), T, M, E, K, F, N, p(Y), o_dtype, p(ws), size(ws_bytes), p(0))


@pytest.mark.parametrize("call,bad", [
    (route, dict(logits=0)), (route, dict(dtype=2)), (route, dict(ldl=63)), (route, dict(T=-1)), (route, dict(E=0)), (route, dict(top=0)), (route, dict(top=65)),
    (route, dict(chosen=0)), (route, dict(share=0)), (route, dict(rows=0)), (route, dict(place=0)), (route, dict(offsets=0)), (route, dict(row_share=0)),
    (combine, dict(y=0)), (combine, dict(dtype=3)), (combine, dict(place=0)), (combine, dict(share=0)), (combine, dict(T=-1)), (combine, dict(top=0)),
    (combine, dict(M=-1)), (combine, dict(N=0)), (combine, dict(out=0)), (combine, dict(o_dtype=-1)), (combine, dict(out=B + 2)), (combine, dict(y=A + 1, dtype=BF16)),
    (combine, dict(residual=R, ldr=63)), (combine, dict(residual=R, r_dtype=7)), (combine, dict(residual=B + 4)), (combine, dict(residual=B, ldr=68)),
    (combine, dict(out=A, o_dtype=F32)), (combine, dict(y=B + 4 * 64 * 4 - 4)), (combine, dict(y=B - 8 * 64 * 4 + 4)),
    (layer, dict(X=0)), (layer, dict(X=ODD)), (layer, dict(dtype=5)), (layer, dict(ldx=255)), (layer, dict(ldx=260)), (layer, dict(rows=0)), (layer, dict(share=0)),
    (layer, dict(offsets=0)), (layer, dict(up=0)), (layer, dict(up=ODD)), (layer, dict(up_s=0)), (layer, dict(down=0)), (layer, dict(down=ODD)), (layer, dict(down_s=0)),
    (layer, dict(residual=R, ldr=63)), (layer, dict(residual=B + 2)), (layer, dict(T=-1)), (layer, dict(M=-1)), (layer, dict(E=0)), (layer, dict(K=0)), (layer, dict(F=0)),
    (layer, dict(N=0)), (layer, dict(Y=0)), (layer, dict(Y=B + 1)), (layer, dict(o_dtype=2)),
])
def test_invalid_arguments(st, call, bad):  # noqa: F811
    assert call(st, **bad) == INVALID
    assert st.stamp_last_launch_count() == 0


@pytest.mark.parametrize("call,bad", [
    (route, dict(E=1025, ldl=1025)), (route, dict(top=33)), (route, dict(T=1 << 28)), (route, dict(ldl=1 << 60)),
    (combine, dict(N=1 << 24, ldr=1 << 24)), (combine, dict(residual=R, ldr=1 << 60)),
    (layer, dict(T=65)), (layer, dict(M=2049)), (layer, dict(E=1025)), (layer, dict(K=100)), (layer, dict(F=24)), (layer, dict(E=1024, F=1 << 20)),
    (layer, dict(E=1024, N=1 << 21)), (layer, dict(K=(1 << 31) - 16)), (layer, dict(ldx=1 << 60)), (layer, dict(residual=R, ldr=1 << 60)),
])
def test_unsupported_sizes(st, call, bad):  # noqa: F811
    assert call(st, **bad) == UNSUPPORTED
    assert st.stamp_last_launch_count() == 0


@pytest.mark.parametrize("call,bad", [
    (route, dict(T=129)), (route, dict(T=4096, ws=A, ws_bytes=100)), (route, dict(T=4096, ws=A + 16, ws_bytes=1 << 20)),
    (layer, dict(ws=0)), (layer, dict(ws=A + 16)), (layer, dict(ws_bytes=8 * 128 * 4 - 1)),
])
def test_workspaces_are_checked(st, call, bad):  # noqa: F811
    assert call(st, **bad) == WORKSPACE
    assert st.stamp_last_launch_count() == 0


def test_workspace_sizes(st):  # noqa: F811
    out = size(7)
    f = st.lib().stamp_expert_route_workspace_bytes
    assert f(128, 64, 8, ctypes.byref(out)) == OK and out.value == 0
    assert f(4096, 64, 8, ctypes.byref(out)) == OK and out.value >= 64 * 4 and out.value % 256 == 0
    assert f(4, 64, 65, ctypes.byref(out)) == INVALID and f(4, 1025, 8, ctypes.byref(out)) == UNSUPPORTED and f(4, 64, 8, None) == INVALID
    f = st.lib().stamp_fp8_expert_workspace_bytes
    assert f(8, 128, ctypes.byref(out)) == OK and out.value >= 8 * 128 * 4 and out.value % 256 == 0
    assert f(0, 128, ctypes.byref(out)) == OK
    assert f(-1, 128, ctypes.byref(out)) == INVALID and f(2049, 128, ctypes.byref(out)) == UNSUPPORTED and f(8, 0, ctypes.byref(out)) == INVALID and f(8, 128, None) == INVALID


def test_no_tokens_launch_nothing(st):  # noqa: F811
    assert combine(st, T=0, place=0, share=0, out=0) == OK
    assert layer(st, T=0, M=0, X=0, Y=0, rows=0, share=0, ws=0) == OK
    assert st.stamp_last_launch_count() == 0


def test_the_marshalling_module_refuses_what_is_not_a_cuda_tensor(st):  # noqa: F811
    import torch
    x, i = torch.zeros(4, 16), torch.zeros(4, 2, dtype=torch.int32)
    c, s = torch.zeros(1, 16, 16).to(torch.float8_e4m3fn), torch.zeros(1, 1, 1, dtype=torch.uint8).view(torch.float8_e8m0fnu)
    for bad in (lambda: st.stamp_expert_route(x, 2), lambda: st.stamp_expert_route(None, 2), lambda: st.stamp_expert_combine(x, i, i.float()),
                lambda: st.stamp_expert_combine(3, i, i.float()), lambda: st.stamp_fp8_expert_layer(x, i[0], i[0].float(), i[0], c, s, c, s),
                lambda: st.calls().expert_route(x), lambda: st.calls().expert_combine(x), lambda: st.calls().fp8_expert_layer(x)):
        with pytest.raises(ValueError):
            bad()


FAR, Y = 1 << 40, 1 << 41
SIX = dict(zip(("chosen", "share", "rows", "place", "offsets", "row_share"), (FAR + (i << 20) for i in range(6))))


# Other CTAs, and the second kernel, may still read what one writes: outputs and scratch share no memory with each other nor with
# what is read meanwhile.
@pytest.mark.parametrize("call,bad", [
    *((route, {a: SIX[b]}) for a in SIX for b in SIX if a < b), (route, dict(rows=SIX["place"] + 4 * 8 * 4 - 4)), (route, dict(offsets=SIX["share"] - 64 * 4)),
    *((route, {a: A + 4 * 64 * 4 - 4}) for a in SIX), (route, dict(T=4096, ws=SIX["rows"], ws_bytes=1 << 20)), (route, dict(T=4096, ws=A, ws_bytes=1 << 20)),
    (combine, dict(place=B)), (combine, dict(place=B - 4 * 2 * 4 + 4)), (combine, dict(share=B + 4 * 64 * 4 - 4)),
    *((layer, {a: Y}) for a in ("rows", "share", "offsets", "down", "down_s", "down_b", "ws")), (layer, dict(offsets=Y - 12)), (layer, dict(ws=Y - 4096)),
    *((layer, {a: FAR}) for a in ("X", "rows", "share", "offsets", "up", "up_s", "up_b", "down", "down_s", "down_b", "residual")),
])
def test_outputs_over_what_is_read_are_refused(st, call, bad):  # noqa: F811
    assert call(st, **{**(SIX if call is route else dict(Y=Y, ws=FAR) if call is layer else {}), **bad}) == INVALID
    assert st.stamp_last_launch_count() == 0


@pytest.mark.parametrize("T,M,E,K,F,dtype,up", [(1, 4, 16, 1152, 2048, "bfloat16", 1), (1, 4, 16, 4096, 512, "bfloat16", 4), (1, 1, 8, 1024, 512, "float32", 8),
                                                (64, 512, 8, 4096, 512, "bfloat16", 1), (64, 512, 8, 4096, 512, "float32", 1), (64, 512, 8, 2048, 256, "bfloat16", 1),
                                                (64, 64, 1, 4096, 1024, "bfloat16", 4), (64, 64, 1, 4096, 1024, "float32", 1), (64, 128, 2, 4096, 128, "bfloat16", 8),
                                                (64, 128, 2, 4096, 128, "float32", 4), (64, 512, 64, 2048, 2048, "bfloat16", 1)])
def test_tiles_of_the_first_kernel_are_shared_where_they_are_few(st, T, M, E, K, F, dtype, up):  # noqa: F811
    """A tile is 128 channels of one run, and an expert's rows make a run for every 16 (fp32 tokens: 8) of them: a cluster takes one
    tile only, so that many short rounds of whole SMs would come of counting experts instead (on 148 SMs)."""
    import torch
    assert st.stamp_debug_expert_plan(T, M, E, K, F, K, dtype=getattr(torch, dtype))[0] == up


@pytest.mark.parametrize("tiles,down", [(5, 16), (12, 16), (13, 10), (16, 10), (23, 10), (24, 9), (26, 9), (27, 8), (28, 8), (29, 8), (30, 7), (32, 7), (33, 7), (34, 6),
                                        (39, 6), (40, 5), (47, 5), (48, 4), (59, 4), (60, 3), (78, 3), (79, 2), (118, 2), (119, 1)])
def test_ctas_of_the_second_kernels_tiles(st, tiles, down):  # noqa: F811
    """The rule where every CTA has enough to do: as many to a tile as leave 1.6 CTAs an SM at most (on 148 SMs)."""
    for T, M, E, F in ((13, 52, 32, 4096), (64, 512, 64, 2048), (55, 440, 8, 3456)):
        assert st.stamp_debug_expert_plan(T, M, E, 1024, F, 128 * tiles)[1] == down
    # little to do: one CTA an SM
    split = 1
    while split < 8 and tiles * split * 2 <= 148:
        split *= 2
    assert st.stamp_debug_expert_plan(1, 1, 16, 1024, 256, 128 * tiles)[1] == split


def test_plans_of_what_is_refused(st):  # noqa: F811
    out = [ctypes.byref(ctypes.c_int()) for _ in range(2)]
    f = st.lib().stamp_debug_expert_plan
    assert f(4, 8, 3, 256, 128, 64, BF16, *out) == OK and f(4, 8, 3, 256, 128, 64, BF16, None, out[1]) == INVALID
    assert f(4, 0, 3, 256, 128, 64, BF16, *out) == INVALID and f(4, 8, 3, 256, 128, 64, 2, *out) == INVALID and f(65, 8, 3, 256, 128, 64, BF16, *out) == UNSUPPORTED
