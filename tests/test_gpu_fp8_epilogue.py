"""The block-scaled product with bias, activation and residual in its epilogue, and with quantized outputs, against plain
statements in 64 bits.

Tolerances, derived before the first run:
  sum         as for the plain product: off = K * 2^-23 * sum_k |x_k w_k| (+ |bias| 2^-24).
  activation  its slope is at most 1.13 (gelu; silu 1.10, relu 1), so the sum's error comes out 1.13 times as large at most.
              Its own error, relative to its value: silu 4 ulp = 2^-21; gelu: the scaled complementary error function within
              2^-21, the exponential within 2 ulp = 2^-22, three products of half an ulp: 2^-20; gelu_tanh: 2 u is a product of three roundings and two rounded constants, at most 5 * 2^-24 of
              itself, which the exponential turns into |2 u| times that; power, sum and quotient add at most 3 ulp each:
              (5 |2 u| + 18) * 2^-24.  Values below 1e-36 may be flushed.
  residual    one addition: 2^-24 of the result.
  output      half the distance of two neighbours of its type (8 significant bits for bf16, 24 for fp32).
  quantized   the scale is that of the exact values unless their largest magnitude lies within its error of the border
              between two scales; a code is within half a step of value / scale, plus the value's error / scale.
With small integer operands every sum is exact in fp32: there, without an activation or with relu, outputs, codes and scales
are equal to those of the definition bit for bit."""
import math

import numpy as np
import pytest

from .test_gpu_fp8 import BLOCK, codes_of, plain_quantize, same, st, values, weights_of  # noqa: F401
from .test_gpu_fp8_plans import Exact

pytestmark = pytest.mark.gpu

ACTS = ["none", "relu", "gelu", "gelu_tanh", "silu"]


def act_code(st, name):  # noqa: F811
    return getattr(st, "ACT_" + name.upper())


def plain_activation(z, name):
    """z in fp64, with the relative error its fp32 form may have."""
    if name == "relu":
        return np.where(z < 0, 0.0, z), np.zeros_like(z)
    if name == "gelu":
        from scipy.special import ndtr
        return z * ndtr(z), np.full_like(z, 2.0 ** -20)
    if name == "gelu_tanh":
        two_u = 2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)
        return z * np.exp(-np.logaddexp(0.0, -two_u)), (5 * np.abs(two_u) + 18) * 2.0 ** -24
    if name == "silu":
        return z * np.exp(-np.logaddexp(0.0, -z)), np.full_like(z, 2.0 ** -21)
    return z, np.zeros_like(z)


def expected(x, w, bias, act):
    """Values before the residual in 64 bits and how far an fp32 evaluation may be off."""
    z, room = x @ w.T, np.abs(x) @ np.abs(w).T
    if bias is not None:
        z, room = z + bias, room + np.abs(bias)
    y, relative = plain_activation(z, act)
    return y, 1.13 * x.shape[1] * 2.0 ** -23 * room + relative * np.abs(y) + 1e-36


def check(y, want, off, residual=None):
    if residual is not None:
        want = want + residual
    off = off + 2.0 ** -24 * np.abs(want)
    bits = 8 if str(y.dtype) == "torch.bfloat16" else 24
    bound = off + 2.0 ** (np.floor(np.log2(np.abs(want) + off)) - bits)
    got = y.double().cpu().numpy()
    bad = ~(np.abs(got - want) <= bound)
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:5].tolist(), float(np.max(np.abs(got - want) / bound)))


def operands(st, M, K, N, seed=0):  # noqa: F811
    """Codes whose products are around one, so that the activations' bends are met."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    x, xs = st.stamp_fp8_quantize(torch.randn(M, K, generator=g, device="cuda").bfloat16())
    w, ws = st.stamp_fp8_quantize_weights(2.0 * torch.randn(N, K, generator=g, device="cuda") * K ** -0.5)
    return x, xs, w, ws, torch.randn(N, generator=g, device="cuda")


# one CTA, a split sum, pairs; odd rows and channels; a short last block
SIZES = [(1, 16, 1), (1, 4096, 130), (3, 400, 257), (33, 1152, 640), (129, 272, 513), (300, 640, 1000), (777, 512, 1160), (700, 4224, 384)]


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("M,K,N", SIZES)
def test_against_the_definition(st, M, K, N, act):  # noqa: F811
    import torch
    x, xs, w, ws, bias = operands(st, M, K, N, seed=M + N)
    want, off = expected(values(x, xs), values(w, ws, True), bias.double().cpu().numpy(), act)
    for out in (torch.bfloat16, torch.float32):
        for residual in (None, 3 * torch.randn(M, N, device="cuda", dtype=torch.bfloat16), torch.randn(M, N, device="cuda")):
            y = st.stamp_fp8_linear_fused(x, xs, w, ws, bias=bias, activation=act_code(st, act), residual=residual, out_dtype=out)
            assert y.dtype == out
            check(y, want, off, None if residual is None else residual.double().cpu().numpy())
    assert st.stamp_last_device_status() == 0


def check_quantized(codes, scale, want, off):
    c, s = codes.double().cpu().numpy(), scale.double().cpu().numpy()
    M, N = want.shape
    nb = -(-N // BLOCK)
    assert c.shape == want.shape and s.shape == (M, nb)
    pad = lambda a: np.pad(a, ((0, 0), (0, nb * BLOCK - N))).reshape(M, nb, BLOCK)  # noqa: E731
    low, high = np.max(pad(np.maximum(np.abs(want) - off, 0)), axis=2), np.max(pad(np.abs(want) + off), axis=2)
    # the smallest power of two that holds: of some maximum between low and high
    assert (low <= 448 * s).all() and ((high > 224 * s) | (s == 2.0 ** -126) | ((s == 1) & (low == 0))).all()
    at = np.repeat(s, BLOCK, axis=1)[:, :N]
    v, err = want / at, off / at
    step = 2.0 ** (np.maximum(np.floor(np.log2(np.abs(v) + err + 1e-300)), -6) - 3)
    bad = ~(np.abs(c - v) <= 0.5 * step + err)
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:5].tolist())


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("M,K,N", [(1, 16, 16), (1, 4096, 144), (3, 400, 272), (33, 1152, 640), (129, 272, 512), (300, 640, 1008), (777, 512, 1168), (2, 14336, 128)])
def test_quantized_against_the_definition(st, M, K, N, act):  # noqa: F811
    x, xs, w, ws, bias = operands(st, M, K, N, seed=M + N)
    want, off = expected(values(x, xs), values(w, ws, True), bias.double().cpu().numpy(), act)
    codes, scale = st.stamp_fp8_linear_quantized(x, xs, w, ws, bias=bias, activation=act_code(st, act))
    check_quantized(codes, scale, want, off)
    assert st.stamp_last_device_status() == 0


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("M,K,N", [(3000, 640, 4112), (2300, 1024, 4112), (1700, 2048, 4096)])
def test_quantized_pairs_against_the_definition(st, M, K, N, act):  # noqa: F811
    assert st.stamp_debug_fp8_plan(M, N, K)[0]
    x, xs, w, ws, bias = operands(st, M, K, N, seed=M + N)
    want, off = expected(values(x, xs), values(w, ws, True), bias.double().cpu().numpy(), act)
    for _ in range(2):
        codes, scale = st.stamp_fp8_linear_quantized(x, xs, w, ws, bias=bias, activation=act_code(st, act))
        check_quantized(codes, scale, want, off)
    assert st.stamp_last_device_status() == 0


# every kernel: single CTAs of each height, sums split by 2, 4 and 8, pairs of several heights; outputs that the tiles do not fill
PLANS = [(1, 512, 128), (16, 4096, 512), (5, 2048, 130), (64, 4096, 384), (100, 1024, 2000), (512, 1024, 4096), (777, 2064, 4104), (1024, 640, 4096),
         (2048, 512, 4096), (1500, 1040, 11008), (4096, 256, 1152), (8, 8192, 64)]


@pytest.mark.parametrize("M,K,N", PLANS)
def test_integers_come_out_exact(st, M, K, N):  # noqa: F811
    import torch
    e = Exact(M, K, N, bias=True, seed=3)
    residual = torch.randint(-50, 51, (M, N), device="cuda").float()
    for act in ("none", "relu"):
        y = e.value if act == "none" else e.value.clamp(min=0)
        for out in (torch.float32, torch.bfloat16):
            for r in (None, residual, residual.bfloat16()):
                got = st.stamp_fp8_linear_fused(e.x, e.xs, e.w, e.ws, bias=e.bias, activation=act_code(st, act), residual=r, out_dtype=out)
                want = (y if r is None else y + r.double()).float().to(out)
                assert torch.equal(got, want), (act, out)
    assert st.stamp_last_device_status() == 0


@pytest.mark.parametrize("M,K,N", [(M, K, N // 16 * 16) for M, K, N in PLANS])
def test_quantized_integers_come_out_exact(st, M, K, N):  # noqa: F811
    import torch
    e = Exact(M, K, N, bias=True, seed=4)
    for act in ("none", "relu"):
        y = (e.value if act == "none" else e.value.clamp(min=0)).float()
        # (the quantizer of fp32 rows is tested against its definition bit for bit)
        want, want_scale = st.stamp_fp8_quantize(y)
        codes = torch.full((M, N), 0x7F, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
        scale = torch.full((M, -(-N // BLOCK)), 0xFF, dtype=torch.uint8, device="cuda").view(torch.float8_e8m0fnu)
        got = st.stamp_fp8_linear_quantized(e.x, e.xs, e.w, e.ws, bias=e.bias, activation=act_code(st, act), codes=codes, scale=scale)
        assert got[0] is codes or got[0].data_ptr() == codes.data_ptr()
        assert torch.equal(scale.view(torch.uint8), want_scale.view(torch.uint8))
        assert torch.equal(codes.float(), want.float())
    assert st.stamp_last_device_status() == 0


@pytest.mark.parametrize("K,spread,error", [(4096, False, 4.4e-7), (14336, False, 4.4e-7), (4096, True, 3.3e-6), (14336, True, 3.3e-6)])
@pytest.mark.parametrize("M,N", [(1024, 4096), (200, 528)])
def test_long_quantized_sums_are_as_near_as_stated(st, M, N, K, spread, error):  # noqa: F811
    """What the header says of the sums, for the inputs it names, as a share of the outputs' root mean square; no single
    sum is taken to be further off than eight times that."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(K + N)
    x = torch.randn(M, K, generator=g, device="cuda")
    x *= torch.where(torch.rand(K, generator=g, device="cuda") < 0.01, 30.0, 1.0)
    w = 0.02 * torch.randn(N, K, generator=g, device="cuda")
    x, xs = st.stamp_fp8_quantize(x)
    w, ws = st.stamp_fp8_quantize_weights(w)
    if spread:
        xs = (torch.randint(-7, 3, xs.shape, generator=g, device="cuda") + 127).to(torch.uint8).view(torch.float8_e8m0fnu)
    exact = lambda c, s, rows: c.double() * s.double().repeat_interleave(BLOCK, 1)[:, :K].repeat_interleave(rows, 0)[:c.shape[0]]  # noqa: E731
    want = exact(x, xs, 1) @ exact(w, ws, BLOCK).t()
    off = torch.full_like(want, 8 * error * float(want.square().mean().sqrt()))
    codes, scale = st.stamp_fp8_linear_quantized(x, xs, w, ws)
    check_quantized(codes, scale, want.cpu().numpy(), off.cpu().numpy())
    assert st.stamp_last_device_status() == 0


# one CTA, a split sum, single CTAs of 128 rows, pairs; last parts of 16, 128, 512 and 4096 features; last blocks of 16 and 64 channels
@pytest.mark.parametrize("act", ["none", "relu", "gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("M,K,N", [(1, 4096, 144), (1, 14336, 256), (9, 4112, 4112), (40, 11008, 1040), (140, 4224, 528), (300, 4608, 12288), (513, 8192, 4160),
                                   (777, 4112, 4112), (1024, 14336, 2048), (2048, 4608, 4096), (700, 8704, 272), (64, 512, 640), (1700, 1152, 4608), (2300, 2048, 4112)])
def test_quantized_outputs_are_those_of_the_fp32_product(st, M, K, N, act):  # noqa: F811
    """The quantizer's codes and scales of stamp_fp8_linear_fused's fp32 outputs, however long the sum, bit for bit."""
    import torch
    x, xs, w, ws, bias = operands(st, M, K, N, seed=K)
    for b in (None, bias):
        want, want_scale = st.stamp_fp8_quantize(st.stamp_fp8_linear_fused(x, xs, w, ws, bias=b, activation=act_code(st, act), out_dtype=torch.float32))
        for _ in range(2):
            codes = torch.full((M, N), 0x7F, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
            scale = torch.full((M, -(-N // BLOCK)), 0xFF, dtype=torch.uint8, device="cuda").view(torch.float8_e8m0fnu)
            st.stamp_fp8_linear_quantized(x, xs, w, ws, bias=b, activation=act_code(st, act), codes=codes, scale=scale)
            assert torch.equal(scale.view(torch.uint8), want_scale.view(torch.uint8)) and torch.equal(codes.view(torch.uint8), want.view(torch.uint8))
    assert st.stamp_last_device_status() == 0


@pytest.mark.parametrize("M,N", [(512, 4096), (40, 144)])
def test_long_quantized_sums_that_are_not_finite(st, M, N):  # noqa: F811
    """A block of NaN in the first part, the second and the last."""
    import torch
    x, xs, w, ws, bias = operands(st, M, 8704, N, seed=5)
    clean, clean_scale = st.stamp_fp8_linear_quantized(x, xs, w, ws, bias=bias)
    for row, block in ((1, 0), (17, 40), (M - 1, 67)):
        bad = xs.clone()
        bad.view(torch.uint8)[row, block] = 255
        codes, scale = st.stamp_fp8_linear_quantized(x, bad, w, ws, bias=bias)
        others = [m for m in range(M) if m != row]
        assert bool(torch.isnan(codes[row].float()).all()) and bool((scale.view(torch.uint8)[row] == 255).all())
        assert torch.equal(codes[others].view(torch.uint8), clean[others].view(torch.uint8)) and torch.equal(scale[others].view(torch.uint8), clean_scale[others].view(torch.uint8))


@pytest.mark.parametrize("K", [4096, 4224, 8704, 14336])
@pytest.mark.parametrize("M,N", [(777, 4104), (1024, 4096), (140, 520)])
def test_long_fp32_sums_are_activated_once(st, M, N, K):  # noqa: F811
    """fp32 sums of more than 4096 features are kept in the output part by part: activation and residual come once."""
    import torch
    e = Exact(M, K, N, bias=True, seed=5)
    residual = torch.randint(-50, 51, (M, N), device="cuda").float()
    for _ in range(3):
        got = st.stamp_fp8_linear_fused(e.x, e.xs, e.w, e.ws, bias=e.bias, activation=st.ACT_RELU, residual=residual, out_dtype=torch.float32)
        assert torch.equal(got, (e.value.clamp(min=0) + residual.double()).float())
        y = residual.clone()                                                          # in place
        st.stamp_fp8_linear_fused(e.x, e.xs, e.w, e.ws, bias=e.bias, residual=y, out=y)
        assert torch.equal(y, (e.value + residual.double()).float())


@pytest.mark.parametrize("M,K,N", [(1, 512, 128), (9, 4096, 130), (70, 640, 257), (700, 512, 1160)])
@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
def test_the_residual_may_be_updated_in_place(st, M, K, N, dtype):  # noqa: F811
    import torch
    e = Exact(M, K, N, seed=6)
    residual = torch.randint(-50, 51, (M, N), device="cuda").to(getattr(torch, dtype))
    for act in ("none", "relu"):
        want = ((e.value if act == "none" else e.value.clamp(min=0)) + residual.double()).float().to(residual.dtype)
        y = residual.clone()
        assert st.stamp_fp8_linear_fused(e.x, e.xs, e.w, e.ws, activation=act_code(st, act), residual=y, out=y).data_ptr() == y.data_ptr()
        assert torch.equal(y, want)


@pytest.mark.parametrize("M,N", [(3, 130), (40, 66), (200, 384), (700, 1160)])
@pytest.mark.parametrize("shift", [0, 1, 2, 3])
def test_residuals_of_a_wider_matrix_and_off_the_alignment(st, M, N, shift):  # noqa: F811
    import torch
    e = Exact(M, 256, N, seed=7)
    for dtype in (torch.bfloat16, torch.float32):
        for width in (N + 5, N + 8):
            wide = torch.randint(-50, 51, (M, width), device="cuda").to(dtype)
            part = wide[:, shift:shift + N]
            for out in (torch.bfloat16, torch.float32):
                want = (e.value + part.double()).float().to(out)
                assert torch.equal(st.stamp_fp8_linear_fused(e.x, e.xs, e.w, e.ws, residual=part, out_dtype=out), want)
                # an output one element off the vectors' alignment
                y = torch.zeros(M * N + shift, dtype=out, device="cuda")[shift:].view(M, N)
                assert torch.equal(st.stamp_fp8_linear_fused(e.x, e.xs, e.w, e.ws, residual=part, out=y), want)


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("M", [3, 40, 700])
def test_non_finite_values_show_in_their_rows_only(st, M, act):  # noqa: F811
    import torch
    x, xs, w, ws, bias = operands(st, M, 512, 384, seed=M)
    clean = st.stamp_fp8_linear_fused(x, xs, w, ws, bias=bias, activation=act_code(st, act))
    c0, s0 = st.stamp_fp8_linear_quantized(x, xs, w, ws, bias=bias, activation=act_code(st, act))
    xs.view(torch.uint8)[1, 2] = 255                                      # a block that held an infinity or a NaN
    y = st.stamp_fp8_linear_fused(x, xs, w, ws, bias=bias, activation=act_code(st, act))
    c, s = st.stamp_fp8_linear_quantized(x, xs, w, ws, bias=bias, activation=act_code(st, act))
    others = [i for i in range(M) if i != 1]
    assert bool(torch.isnan(y[1]).all()) and torch.equal(y[others], clean[others])
    assert bool(torch.isnan(c[1].float()).all()) and bool((s.view(torch.uint8)[1] == 255).all())
    assert torch.equal(c[others].float(), c0[others].float()) and torch.equal(s.view(torch.uint8)[others], s0.view(torch.uint8)[others])


@pytest.mark.parametrize("act", ACTS)
def test_activations_at_the_ends_of_their_range(st, act):  # noqa: F811
    """x = 1, w = 1, and a bias that is the argument less one: from -1e4 to 1e4, around zero, and where the tails vanish."""
    import torch
    z = np.concatenate([np.linspace(-1e4, 1e4, 41), np.linspace(-95, 95, 761), np.linspace(-1, 1, 201), [-1e20, 1e20, 2e-30, -2e-30]]).astype(np.float32)
    N = len(z)
    x, w = torch.zeros(1, 16, device="cuda"), torch.zeros(N, 16, device="cuda")
    xc, xs = st.stamp_fp8_quantize(x)
    wc, ws = st.stamp_fp8_quantize_weights(w)
    y = st.stamp_fp8_linear_fused(xc, xs, wc, ws, bias=torch.from_numpy(z).cuda(), activation=act_code(st, act), out_dtype=torch.float32)
    want, relative = plain_activation(z.astype(np.float64), act)
    check(y, want[None], (relative * np.abs(want) + 1e-36)[None])


@pytest.mark.parametrize("M,N", [(5, 144), (130, 272), (700, 528)])
def test_no_write_leaves_the_outputs(st, M, N):  # noqa: F811
    import torch
    x, xs, w, ws, bias = operands(st, M, 256, N, seed=1)
    room = torch.full((M * N + 512,), 0xA5, dtype=torch.uint8, device="cuda")
    scales = torch.full((M * -(-N // BLOCK) + 512,), 0xA5, dtype=torch.uint8, device="cuda")
    codes = room[256:256 + M * N].view(torch.float8_e4m3fn).view(M, N)
    scale = scales[256:256 + M * -(-N // BLOCK)].view(torch.float8_e8m0fnu).view(M, -1)
    st.stamp_fp8_linear_quantized(x, xs, w, ws, bias=bias, codes=codes, scale=scale)
    for t in (room, scales):
        assert bool((t[:256] == 0xA5).all()) and bool((t[-256:] == 0xA5).all())
    for dtype in (torch.float32, torch.bfloat16):
        wide = torch.full((M * N + 512,), 7.0, dtype=dtype, device="cuda")
        st.stamp_fp8_linear_fused(x, xs, w, ws, residual=torch.zeros(M, N, dtype=dtype, device="cuda"), out=wide[256:256 + M * N].view(M, N))
        assert bool((wide[:256] == 7).all()) and bool((wide[-256:] == 7).all())


@pytest.mark.parametrize("M", [1, 60, 600])
def test_results_repeat_bit_for_bit_on_other_streams(st, M):  # noqa: F811
    import torch
    x, xs, w, ws, bias = operands(st, M, 4096, 528, seed=3)
    first = st.stamp_fp8_linear_quantized(x, xs, w, ws, bias=bias, activation=st.ACT_GELU)
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(other):
        again = [st.stamp_fp8_linear_quantized(x, xs, w, ws, bias=bias, activation=st.ACT_GELU) for _ in range(4)]
    torch.cuda.current_stream().wait_stream(other)
    assert all(torch.equal(first[0].view(torch.uint8), a[0].view(torch.uint8)) and torch.equal(first[1].view(torch.uint8), a[1].view(torch.uint8)) for a in again)


def test_an_mlp_of_two_kernels_can_be_captured(st):  # noqa: F811
    """Up with gelu and quantized outputs, down with the residual in place: two kernels, captured and replayed on new inputs."""
    import torch
    M, K, F = 40, 512, 1024
    x, xs, up, up_s, b1 = operands(st, M, K, F, seed=8)
    _, _, down, down_s, b2 = operands(st, 1, F, K, seed=9)
    stream = torch.randn(M, K, device="cuda").bfloat16()
    start = stream.clone()

    def mlp(y):
        c, s = st.stamp_fp8_linear_quantized(x, xs, up, up_s, bias=b1, activation=st.ACT_GELU)
        launches = st.stamp_last_launch_count()
        st.stamp_fp8_linear_fused(c, s, down, down_s, bias=b2, residual=y, out=y)
        assert launches == 1 and st.stamp_last_launch_count() == 1
        return c, s

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        mlp(stream.clone())
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        mlp(stream)
    stream.copy_(start)
    xc, xsc = codes_of(st, M, K, seed=10)
    x.copy_(xc)
    xs.copy_(xsc)
    graph.replay()
    want = start.clone()
    c, s = mlp(want)
    assert torch.equal(stream, want)
    y, off = expected(values(c, s), values(down, down_s, True), b2.double().cpu().numpy(), "none")
    check(want, y, off, start.double().cpu().numpy())
    assert st.stamp_last_device_status() == 0


def test_quantized_outputs_of_a_product_feed_the_next(st):  # noqa: F811
    """The same numbers as the product and the quantizer of its fp32 outputs one after the other."""
    import torch
    for M in (1, 50, 900):
        e = Exact(M, 768, 640, seed=11)
        y = st.stamp_fp8_linear(e.x, e.xs, e.w, e.ws, out_dtype=torch.float32)
        c, s = st.stamp_fp8_quantize(y)
        got = st.stamp_fp8_linear_quantized(e.x, e.xs, e.w, e.ws)
        assert torch.equal(got[0].float(), c.float()) and torch.equal(got[1].view(torch.uint8), s.view(torch.uint8))


def test_rows_and_zero_rows(st):  # noqa: F811
    import torch
    w, ws = weights_of(st, (64, 256), seed=1)
    x, xs = torch.empty(0, 256, device="cuda").to(torch.float8_e4m3fn), torch.empty(0, 2, dtype=torch.uint8, device="cuda").view(torch.float8_e8m0fnu)
    assert st.stamp_fp8_linear_fused(x, xs, w, ws, residual=torch.empty(0, 64, device="cuda")).shape == (0, 64)
    c, s = st.stamp_fp8_linear_quantized(x, xs, w, ws)
    assert c.shape == (0, 64) and s.shape == (0, 1) and st.stamp_last_launch_count() == 0


def test_arguments_are_checked(st):  # noqa: F811
    import torch
    x, xs = codes_of(st, 8, 256, seed=1)
    w, ws = weights_of(st, (40, 256), seed=1)
    r = torch.zeros(8, 40, device="cuda")
    for bad in (lambda: st.stamp_fp8_linear_fused(x, xs, w, ws, activation=-1), lambda: st.stamp_fp8_linear_fused(x, xs, w, ws, activation="gelu"),
                lambda: st.stamp_fp8_linear_fused(x, xs, w, ws, residual=r[:, :39]), lambda: st.stamp_fp8_linear_fused(x, xs, w, ws, residual=r[:7]),
                lambda: st.stamp_fp8_linear_fused(x, xs, w, ws, residual=r.half()), lambda: st.stamp_fp8_linear_fused(x, xs, w, ws, residual=r.cpu()),
                lambda: st.stamp_fp8_linear_fused(x, xs, w, ws, residual=torch.zeros(40, 8, device="cuda").t()),
                lambda: st.stamp_fp8_linear_fused(x, xs, w, ws, residual=torch.zeros(1, 40, device="cuda").expand(8, 40)),
                lambda: st.stamp_fp8_linear_fused(x, xs, w, ws, out_dtype=torch.float16),
                lambda: st.stamp_fp8_linear_fused(x, xs, w, ws, bias=torch.zeros(39, device="cuda")),
                lambda: st.stamp_fp8_linear_fused(x, xs, w.view(1, 40, 256), ws),
                lambda: st.stamp_fp8_linear_quantized(x, xs, w, ws, codes=torch.zeros(8, 40, device="cuda")),
                lambda: st.stamp_fp8_linear_quantized(x, xs[:, :1].contiguous(), w, ws)):
        with pytest.raises(ValueError):
            bad()
    wide = torch.zeros(8, 80, device="cuda")
    long_x, long_xs = codes_of(st, 8, 4224, seed=1)
    long_w, long_ws = weights_of(st, (40, 4224), seed=1)
    for status, bad in ((1, lambda: st.stamp_fp8_linear_fused(x, xs, w, ws, activation=5)),
                        (1, lambda: st.stamp_fp8_linear_fused(x, xs, w, ws, residual=wide[:, :40], out=wide.view(16, 40)[:8])),      # overlaps
                        (1, lambda: st.stamp_fp8_linear_fused(x, xs, w, ws, residual=r, out=r.view(torch.bfloat16).view(16, 40)[:8])),
                        (1, lambda: st.stamp_fp8_linear_fused(long_x, long_xs, long_w, long_ws, activation=st.ACT_RELU, residual=r, out=r)),
                        (2, lambda: st.stamp_fp8_linear_quantized(x, xs, w, ws))):                                                  # N = 40
        with pytest.raises(st.StampError) as e:
            bad()
        assert e.value.status == status
    assert st.stamp_last_device_status() == 0
