"""The block-scaled 8-bit floating point layers (quantizers, product, product grouped by expert) against plain
statements of their definitions in 64 bits.

Tolerances, derived before the first run:
  quantizer      every step but one is exact (the scale comes from exponent bits, the division by it is exact), and
                 the code's rounding is fixed: codes and scales are equal, bit for bit.
  gated          h = g / (1 + exp(-g)) * u in fp32: expf within 2 ulp, three further roundings -- h is within 4 ulp
                 (2.4e-7 relative) of its value.  A code can then differ only where h / scale is that near a rounding
                 boundary, and by one step.
  product        the codes' products are exact in fp32, a sum of K of them in fp32 has an error of at most
                 K * 2^-24 * sum |terms|; a tensor core may cut terms off where fp32 would round, which doubles the unit:
                 |y - exact| <= K * 2^-23 * sum_k |x_k w_k| + half the distance of two neighbours of the output type
                 there (8 significant bits for bf16, 24 for fp32)."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

BLOCK = 128


@pytest.fixture(scope="module")
def st():
    import torch
    from paper_2510_26771_b200 import binding
    assert torch.cuda.is_available()
    binding.lib()
    return binding


# ------------------------------------------------------------------------------------------ plain statements, numpy fp64
def _blocks(n):
    return -(-n // BLOCK)


def plain_scale(amax):
    """The smallest power of two >= 2^-126 with amax / scale <= 448; 1 for a block of zeros, NaN for a non-finite one."""
    amax = np.asarray(amax, dtype=np.float64)
    out = np.ones_like(amax)
    for i, a in np.ndenumerate(amax):
        if not np.isfinite(a):
            out[i] = np.nan
        elif a > 0:
            s = 2.0 ** -126
            while a / s > 448.0:
                s *= 2.0
            out[i] = s
    return out


def plain_e4m3(v):
    """v rounded to the nearest e4m3 number, ties to even; |v| <= 448."""
    v = np.asarray(v, dtype=np.float64)
    with np.errstate(divide="ignore", invalid="ignore"):
        step = 2.0 ** np.maximum(np.floor(np.log2(np.abs(v))) - 3, -9)
    step = np.where(np.isfinite(step) & (step > 0), step, 2.0 ** -9)
    return np.round(v / step) * step


def plain_quantize(x):
    x = np.asarray(x, dtype=np.float64)
    M, K = x.shape
    nb = _blocks(K)
    p = np.zeros((M, nb * BLOCK))
    p[:, :K] = x
    p = p.reshape(M, nb, BLOCK)
    s = plain_scale(np.max(np.abs(p), axis=2)) if M else np.zeros((0, nb))
    c = np.where(np.isnan(s)[:, :, None], np.nan, plain_e4m3(p / np.where(np.isnan(s), 1.0, s)[:, :, None]))
    return c.reshape(M, nb * BLOCK)[:, :K], s


def values(codes, scale, weights=False):
    """Torch codes and scales -> the fp64 numbers they stand for."""
    c, s = codes.double().cpu().numpy(), scale.double().cpu().numpy()
    s = np.repeat(s, BLOCK, axis=-1)[..., : c.shape[-1]]
    if weights:
        s = np.repeat(s, BLOCK, axis=-2)[..., : c.shape[-2], :]
    return c * s


def check_product(y, x, w, bias=None):
    """y (torch) against x @ w.T (+ bias) in fp64, element by element within the derived bound."""
    want, room = x @ w.T, np.abs(x) @ np.abs(w).T
    if bias is not None:
        want, room = want + bias, room + np.abs(bias)
    off = x.shape[1] * 2.0 ** -23 * room
    bits = 8 if str(y.dtype) == "torch.bfloat16" else 24
    bound = off + 2.0 ** (np.floor(np.log2(np.abs(want) + off + 1e-30)) - bits)
    got = y.double().cpu().numpy()
    assert got.shape == want.shape
    bad = np.abs(got - want) > bound
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:5].tolist(), float(np.max(np.abs(got - want) / bound)))


def same(got, want):
    g = got.double().cpu().numpy()
    return g.shape == want.shape and np.array_equal(g, want, equal_nan=True)


def activations(M, K, dtype, seed=0):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(M, K, generator=g, device="cuda")
    x *= torch.where(torch.rand(K, generator=g, device="cuda") < 0.02, 40.0, 1.0)
    x *= torch.exp2(torch.randint(-12, 12, (M, 1), generator=g, device="cuda").float())
    return x.to(dtype)


def codes_of(st, M, K, seed):
    import torch
    return st.stamp_fp8_quantize(activations(M, K, torch.bfloat16, seed))


def weights_of(st, shape, seed):
    import torch
    g = torch.Generator(device="cuda").manual_seed(1000 + seed)
    w = 0.02 * torch.randn(*shape, generator=g, device="cuda")
    # blocks of very different size, so that a scale taken from a neighbouring block shows
    w *= torch.exp2(torch.randint(-6, 6, (*shape[:-1], 1), generator=g, device="cuda").float())
    return st.stamp_fp8_quantize_weights(w)


# ------------------------------------------------------------------------------------------ quantizers
@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("M,K", [(1, 16), (1, 4096), (3, 128), (7, 144), (33, 1152), (5, 2064), (200, 640), (1, 14336), (129, 48)])
def test_quantizer_codes_and_scales_are_exact(st, M, K, dtype):
    import torch
    x = activations(M, K, getattr(torch, dtype), seed=M + K)
    x[:, : min(K, 8)] *= 0.0                                   # zeros inside a block
    if M > 2:
        x[1] = 0                                               # a row of zeros: scale 1
    codes, scale = st.stamp_fp8_quantize(x)
    c, s = plain_quantize(x.double().cpu().numpy())
    assert codes.dtype == torch.float8_e4m3fn and scale.dtype == torch.float8_e8m0fnu
    assert same(scale, s) and same(codes, c)
    assert st.stamp_last_device_status() == 0


def test_quantizer_at_the_edges_of_the_types(st):
    """Largest and smallest numbers, the boundary between two scales (448 * 2^e and its neighbours), ties between codes,
    infinities and NaN in one block only."""
    import torch
    x = torch.zeros(12, 384, dtype=torch.float32, device="cuda")
    x[0, 5] = 448.0
    x[1, 5] = float(np.nextafter(np.float32(448.0), np.float32(1e9)))
    x[2, 130] = 3.4028234663852886e38
    x[3, 130] = 1e-45                                          # the smallest subnormal: clamped scale, code 0 or its value
    x[4, 0] = 2.0 ** -126 * 448
    x[5, 0] = 2.0 ** -127 * 448
    x[6, :128] = torch.linspace(-448, 448, 128, device="cuda")
    x[7, 0], x[7, 1:17] = 448.0, torch.arange(16, device="cuda") * 2.0 ** -10   # ties among the e4m3 subnormals
    x[8, 200] = float("inf")
    x[8, 0] = 3.0
    x[9, 300] = float("nan")
    x[10, 300] = float("-inf")
    x[11] = -0.0
    codes, scale = st.stamp_fp8_quantize(x)
    c, s = plain_quantize(x.double().cpu().numpy())
    assert same(scale, s) and same(codes, c)
    b, sb = st.stamp_fp8_quantize(x.to(torch.bfloat16))
    c, s = plain_quantize(x.to(torch.bfloat16).double().cpu().numpy())
    assert same(sb, s) and same(b, c)


def test_quantizer_gathers_rows(st):
    import torch
    x = activations(37, 272, torch.bfloat16, seed=3)
    rows = torch.tensor([36, 0, 0, 5, 17, 36, 1] * 9, dtype=torch.int32, device="cuda")
    codes, scale = st.stamp_fp8_quantize(x, rows=rows)
    c, s = plain_quantize(x.double().cpu().numpy()[rows.cpu().numpy()])
    assert same(scale, s) and same(codes, c)
    none, none_scale = st.stamp_fp8_quantize(x, rows=rows[:0])
    assert none.shape == (0, 272) and none_scale.shape == (0, 3)
    assert st.stamp_last_device_status() == 0
    # an index outside the tokens: a row of zeros, reported once
    rows[4], rows[9] = 37, -1
    codes, scale = st.stamp_fp8_quantize(x, rows=rows)
    assert st.stamp_last_device_status() == 1 and st.stamp_last_device_status() == 0
    c, s = plain_quantize(x.double().cpu().numpy()[np.where(rows.cpu().numpy() % 37 == rows.cpu().numpy(), rows.cpu().numpy(), 0)])
    c[[4, 9]], s[[4, 9]] = 0, 1
    assert same(scale, s) and same(codes, c)


def test_quantizer_takes_rows_of_a_wider_matrix(st):
    import torch
    wide = activations(19, 3 * 256 + 64, torch.bfloat16, seed=8)
    x = wide[:, 256:256 + 400]
    codes, scale = st.stamp_fp8_quantize(x)
    c, s = plain_quantize(x.double().cpu().numpy())
    assert same(scale, s) and same(codes, c)
    with pytest.raises(st.StampError):
        st.stamp_fp8_quantize(wide[:, 3:3 + 256])              # rows off the 16-byte boundaries
    with pytest.raises(ValueError):
        st.stamp_fp8_quantize(wide.t())


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("M,F", [(1, 16), (1, 2048), (33, 2048), (7, 400), (130, 1152)])
def test_gated_quantizer(st, M, F, dtype):
    import torch
    x = activations(M, 2 * F, getattr(torch, dtype), seed=F)
    x.clamp_(-3000, 3000)
    x[0, 0], x[0, 1], x[0, 2] = -200.0, 200.0, 0.0             # exp(-g) overflows, vanishes, is one
    codes, scale = st.stamp_fp8_gated_quantize(x)
    v = x.double().cpu().numpy()
    with np.errstate(over="ignore"):
        h = v[:, :F] / (1.0 + np.exp(-v[:, :F])) * v[:, F:]
    c, s = plain_quantize(h)
    got_c, got_s = codes.double().cpu().numpy(), scale.double().cpu().numpy()
    # a scale may differ only where max |h| is within 4 ulp of a boundary (none is here)
    assert np.array_equal(got_s, s)
    lo, hi = (plain_quantize_with(h * (1 - 2.4e-7), s), plain_quantize_with(h * (1 + 2.4e-7), s))
    assert np.all((got_c == c) | (got_c == lo) | (got_c == hi))
    assert np.count_nonzero(got_c != c) <= max(2, 1e-4 * c.size)


def plain_quantize_with(h, s):
    return plain_e4m3(h / np.repeat(s, BLOCK, axis=1)[:, : h.shape[1]])


def test_gated_quantizer_lets_non_finite_blocks_show(st):
    import torch
    x = torch.ones(3, 512, dtype=torch.float32, device="cuda")
    x[0, 3], x[1, 256 + 140], x[2, 0] = float("nan"), float("inf"), float("-inf")   # gate, up, gate: -inf / (1 + inf) is NaN
    codes, scale = st.stamp_fp8_gated_quantize(x)
    assert torch.isnan(scale.float()).tolist() == [[True, False], [False, True], [True, False]]
    assert torch.isnan(codes.float()).view(3, 2, 128).all(dim=2).tolist() == [[True, False], [False, True], [True, False]]


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("shape", [(1, 16), (128, 128), (130, 272), (72, 1152), (3, 129, 144)])
def test_weight_quantizer(st, shape, dtype):
    import torch
    g = torch.Generator(device="cuda").manual_seed(shape[-1])
    w = (torch.randn(*shape, generator=g, device="cuda") * torch.exp2(3 * torch.randn(*shape[:-1], 1, generator=g, device="cuda"))).to(getattr(torch, dtype))
    codes, scale = st.stamp_fp8_quantize_weights(w)
    v = w.double().cpu().numpy().reshape(-1, *shape[-2:])
    nb, kb = _blocks(shape[-2]), _blocks(shape[-1])
    assert tuple(scale.shape) == (*shape[:-2], nb, kb)
    for e in range(v.shape[0]):
        p = np.zeros((nb * BLOCK, kb * BLOCK))
        p[: shape[-2], : shape[-1]] = v[e]
        p = p.reshape(nb, BLOCK, kb, BLOCK)
        s = plain_scale(np.max(np.abs(p), axis=(1, 3)))
        c = plain_e4m3(p / s[:, None, :, None]).reshape(nb * BLOCK, kb * BLOCK)[: shape[-2], : shape[-1]]
        assert np.array_equal(scale.double().cpu().numpy().reshape(-1, nb, kb)[e], s)
        assert np.array_equal(codes.double().cpu().numpy().reshape(-1, *shape[-2:])[e], c)


# ------------------------------------------------------------------------------------------ product
LINEAR = [
    # M, K, N: single tokens, short sums, odd widths, a short last block, tiles that hang over in every direction
    (1, 16, 1), (1, 128, 128), (1, 4096, 1000), (2, 640, 130), (3, 144, 77), (16, 2048, 264), (17, 1152, 1152), (31, 528, 129),
    (64, 4096, 256), (65, 512, 384), (127, 1040, 200), (128, 128, 640), (129, 272, 257), (200, 2064, 513), (256, 1024, 256),
    (257, 1152, 1152), (300, 3008, 384), (513, 640, 1031), (1024, 512, 512), (1500, 4096, 768), (2049, 272, 520),
]


@pytest.mark.parametrize("out", ["bfloat16", "float32"])
@pytest.mark.parametrize("M,K,N", LINEAR)
def test_product_against_the_definition(st, M, K, N, out):
    import torch
    x, xs = codes_of(st, M, K, seed=M + N)
    w, ws = weights_of(st, (N, K), seed=K)
    y = st.stamp_fp8_linear(x, xs, w, ws, out_dtype=getattr(torch, out))
    check_product(y, values(x, xs), values(w, ws, True))
    assert st.stamp_last_device_status() == 0


@pytest.mark.parametrize("M", [1, 40, 700])
def test_product_adds_the_bias(st, M):
    import torch
    x, xs = codes_of(st, M, 656, seed=5)
    w, ws = weights_of(st, (300, 656), seed=5)
    b = torch.randn(300, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    y = st.stamp_fp8_linear(x, xs, w, ws, bias=b, out_dtype=torch.float32)
    check_product(y, values(x, xs), values(w, ws, True), b.double().cpu().numpy())
    # codes of zeros: the bias alone
    z = st.stamp_fp8_linear(torch.zeros_like(x.view(torch.uint8)).view(x.dtype), xs, w, ws, bias=b, out_dtype=torch.float32)
    assert torch.equal(z, b.expand(M, 300))


@pytest.mark.parametrize("M", [1, 5, 200, 1100])
def test_every_block_meets_its_own_scales(st, M):
    """Integer codes and scales that make each block's share of the sum recognisable: exact in fp32, so equal bit for bit."""
    import torch
    K, N = 1040, 272
    nb = _blocks(K)
    x = torch.randint(-3, 4, (M, K), device="cuda", generator=torch.Generator(device="cuda").manual_seed(2)).float()
    w = torch.randint(-3, 4, (N, K), device="cuda", generator=torch.Generator(device="cuda").manual_seed(3)).float()
    sx = (torch.arange(M, device="cuda")[:, None] * 3 + torch.arange(nb, device="cuda")[None, :]) % 4
    sw = (torch.arange(_blocks(N), device="cuda")[:, None] * 2 + torch.arange(nb, device="cuda")[None, :]) % 3
    y = st.stamp_fp8_linear(x.to(torch.float8_e4m3fn), (sx + 127).to(torch.uint8).view(torch.float8_e8m0fnu),
                            w.to(torch.float8_e4m3fn), (sw + 125).to(torch.uint8).view(torch.float8_e8m0fnu), out_dtype=torch.float32)
    xv = x.double() * torch.exp2(sx.double()).repeat_interleave(128, 1)[:, :K]
    wv = w.double() * torch.exp2(sw.double() - 2).repeat_interleave(128, 1)[:, :K].repeat_interleave(128, 0)[:N]
    assert torch.equal(y.double(), xv @ wv.t())


@pytest.mark.parametrize("shift", [0, 1, 2, 3])
@pytest.mark.parametrize("K", [128, 256, 384, 640, 896])
def test_scale_rows_of_every_length_and_alignment(st, K, shift):
    """x_scale rows of one, two, three, five and seven bytes that start anywhere: read as words, as pairs of aligned words in
    the middle of the table, byte by byte at its ends.  Exact in fp32 again."""
    import torch
    M, N, nb = 700, 136, K // 128
    g = torch.Generator(device="cuda").manual_seed(K + shift)
    x = torch.randint(-3, 4, (M, K), device="cuda", generator=g).float()
    w = torch.randint(-3, 4, (N, K), device="cuda", generator=g).float()
    e = torch.randint(0, 4, (M, nb), device="cuda", generator=g)
    raw = torch.zeros(M * nb + 8, dtype=torch.uint8, device="cuda")
    scale = raw[shift:shift + M * nb].view(M, nb)
    scale.copy_((e + 127).to(torch.uint8))
    one = torch.full((_blocks(N), nb), 127, dtype=torch.uint8, device="cuda").view(torch.float8_e8m0fnu)
    want = (x.double() * torch.exp2(e.double()).repeat_interleave(128, 1)) @ w.double().t()
    codes, wc, xs = x.to(torch.float8_e4m3fn), w.to(torch.float8_e4m3fn), scale.view(torch.float8_e8m0fnu)
    assert torch.equal(st.stamp_fp8_linear(codes, xs, wc, one, out_dtype=torch.float32).double(), want)
    offsets = torch.tensor([0, 1, 3, 300, 300, 695, 700], dtype=torch.int32, device="cuda")
    y = st.stamp_fp8_linear_grouped(codes, xs, offsets, wc.view(torch.uint8).expand(6, N, K).contiguous().view(torch.float8_e4m3fn),
                                    one.view(torch.uint8).expand(6, -1, -1).contiguous().view(torch.float8_e8m0fnu), out_dtype=torch.float32)
    assert torch.equal(y.double(), want)


@pytest.mark.parametrize("M", [4, 300])
def test_non_finite_activations_show_in_their_rows_only(st, M):
    import torch
    x = activations(M, 512, torch.bfloat16, seed=2)
    x[1, 300], x[3, 5] = float("inf"), float("nan")
    c, s = st.stamp_fp8_quantize(x)
    w, ws = weights_of(st, (200, 512), seed=4)
    y = st.stamp_fp8_linear(c, s, w, ws)
    bad = torch.zeros(M, dtype=torch.bool, device="cuda")
    bad[1] = bad[3] = True
    assert torch.isnan(y[bad]).all() and torch.isfinite(y[~bad]).all()


def test_zero_rows_launch_nothing(st):
    import torch
    w, ws = weights_of(st, (200, 256), seed=1)
    x, xs = st.stamp_fp8_quantize(torch.empty(0, 256, dtype=torch.bfloat16, device="cuda"))
    assert x.shape == (0, 256) and xs.shape == (0, 2)
    assert st.stamp_fp8_linear(x, xs, w, ws).shape == (0, 200) and st.stamp_last_launch_count() == 0


# ------------------------------------------------------------------------------------------ product grouped by expert
GROUPED = {
    # rows of each expert; K, N
    "one_expert": ([70], 272, 200),
    "one_row_each": ([1] * 9, 1152, 136),
    "empty_runs": ([0, 5, 0, 0, 130, 1, 0], 640, 129),
    "all_empty": ([0, 0, 0], 128, 64),
    "one_takes_all": ([0, 0, 700, 0], 528, 384),
    "ragged": ([33, 257, 1, 128, 0, 64, 300, 17], 1040, 520),
    "large_runs": ([900, 513, 0, 1301], 512, 768),
    "many_experts": ([i % 5 for i in range(200)], 256, 72),
    "most_experts": ([1 if i % 97 == 3 else 0 for i in range(1024)], 128, 128),
}


def grouped_case(st, name, seed=0):
    import torch
    counts, K, N = GROUPED[name]
    M, E = sum(counts), len(counts)
    x, xs = codes_of(st, M, K, seed=seed + 1)
    w, ws = weights_of(st, (E, N, K), seed=seed)
    offsets = torch.tensor(np.concatenate([[0], np.cumsum(counts)]), dtype=torch.int32, device="cuda")
    return x, xs, offsets, w, ws


def check_grouped(y, x, xs, offsets, w, ws, bias=None):
    ends, xv, wv = offsets.tolist(), values(x, xs), values(w, ws, True)
    for e in range(len(ends) - 1):
        if ends[e + 1] > ends[e]:
            rows = slice(ends[e], ends[e + 1])
            check_product(y[rows], xv[rows], wv[e], None if bias is None else bias[e].double().cpu().numpy())


@pytest.mark.parametrize("out", ["bfloat16", "float32"])
@pytest.mark.parametrize("name", list(GROUPED))
def test_grouped_product_against_the_definition(st, name, out):
    import torch
    case = grouped_case(st, name)
    y = st.stamp_fp8_linear_grouped(*case, out_dtype=getattr(torch, out))
    check_grouped(y, *case)
    assert st.stamp_last_device_status() == 0


def test_grouped_product_adds_each_experts_bias(st):
    import torch
    case = grouped_case(st, "ragged", seed=7)
    b = torch.randn(case[3].shape[0], case[3].shape[1], device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    y = st.stamp_fp8_linear_grouped(*case, bias=b, out_dtype=torch.float32)
    check_grouped(y, *case, bias=b)


def test_rows_behind_the_last_run_stay_as_they_were(st):
    import torch
    x, xs, offsets, w, ws = grouped_case(st, "ragged", seed=9)
    offsets = offsets.clone()
    offsets[-1] -= 5
    y = torch.full((x.shape[0], w.shape[1]), 7.0, device="cuda")
    st.stamp_fp8_linear_grouped(x, xs, offsets, w, ws, out=y)
    assert bool((y[-5:] == 7.0).all())
    check_grouped(y, x, xs, offsets, w, ws)


@pytest.mark.parametrize("bad", [[0, 5, 4, 9], [1, 2, 3, 9], [0, 2, 4, 10], [0, -1, 4, 9], [0, 2, 1 << 30, 9]])
def test_offsets_out_of_order_write_nothing_and_are_reported(st, bad):
    import torch
    x, xs = codes_of(st, 9, 256, seed=1)
    w, ws = weights_of(st, (3, 72, 256), seed=1)
    y = torch.full((9, 72), 7.0, device="cuda")
    st.stamp_fp8_linear_grouped(x, xs, torch.tensor(bad, dtype=torch.int32, device="cuda"), w, ws, out=y)
    assert st.stamp_last_device_status() == 1 and st.stamp_last_device_status() == 0
    assert bool((y == 7.0).all())


def test_one_expert_equals_the_plain_product(st):
    import torch
    for M in (3, 200, 900):
        x, xs = codes_of(st, M, 1040, seed=M)
        w, ws = weights_of(st, (1, 392, 1040), seed=M)
        offsets = torch.tensor([0, M], dtype=torch.int32, device="cuda")
        a = st.stamp_fp8_linear_grouped(x, xs, offsets, w, ws, out_dtype=torch.float32)
        check_product(a, values(x, xs), values(w[0], ws[0], True))
        check_product(st.stamp_fp8_linear(x, xs, w[0], ws[0], out_dtype=torch.float32), values(x, xs), values(w[0], ws[0], True))


# ------------------------------------------------------------------------------------------ how they are called
@pytest.mark.parametrize("M,N", [(5, 130), (130, 257), (700, 513)])
@pytest.mark.parametrize("out", ["bfloat16", "float32"])
def test_no_write_leaves_the_outputs(st, M, N, out):
    """Outputs carved out of larger allocations whose margins hold a pattern, at sizes whose tiles hang over every edge."""
    import torch
    dtype = getattr(torch, out)
    K, guard = 528, 4096
    x = activations(M, K, torch.bfloat16, seed=1)
    def room(n):
        return torch.full((n + 2 * guard,), 0x5A, dtype=torch.uint8, device="cuda")
    def intact(raw, n):
        return bool((raw[:guard] == 0x5A).all()) and bool((raw[guard + n:] == 0x5A).all())
    cn, sn, yn = M * K, M * _blocks(K), M * N * (2 if out == "bfloat16" else 4)
    craw, sraw, yraw = room(cn), room(sn), room(yn)
    codes = craw[guard:guard + cn].view(torch.float8_e4m3fn).view(M, K)
    scale = sraw[guard:guard + sn].view(torch.float8_e8m0fnu).view(M, _blocks(K))
    y = yraw[guard:guard + yn].view(dtype).view(M, N)
    st.stamp_fp8_quantize(x, codes=codes, scale=scale)
    w, ws = weights_of(st, (2, N, K), seed=1)
    st.stamp_fp8_linear(codes, scale, w[0], ws[0], out=y)
    st.stamp_fp8_linear_grouped(codes, scale, torch.tensor([0, M // 3, M], dtype=torch.int32, device="cuda"), w, ws, out=y)
    torch.cuda.synchronize()
    assert intact(craw, cn) and intact(sraw, sn) and intact(yraw, yn)


def test_outputs_off_the_vector_alignment(st):
    """An output that starts on an element boundary only (a row of a larger buffer with an odd row length)."""
    import torch
    x, xs = codes_of(st, 70, 256, seed=1)
    w, ws = weights_of(st, (128, 256), seed=1)
    for dtype in (torch.bfloat16, torch.float32):
        raw = torch.zeros(70 * 128 + 8, dtype=dtype, device="cuda")
        y = raw[1:1 + 70 * 128].view(70, 128)
        st.stamp_fp8_linear(x, xs, w, ws, out=y)
        check_product(y, values(x, xs), values(w, ws, True))
        assert raw[0] == 0 and bool((raw[1 + 70 * 128:] == 0).all())


def test_scales_off_the_word_alignment(st):
    """x_scale is read in words where its rows allow that; here it starts on an odd byte."""
    import torch
    x, xs = codes_of(st, 90, 1024, seed=1)
    w, ws = weights_of(st, (136, 1024), seed=1)
    raw = torch.zeros(90 * 8 + 8, dtype=torch.uint8, device="cuda")
    odd = raw[3:3 + 90 * 8].view(torch.float8_e8m0fnu).view(90, 8)
    odd.view(torch.uint8).copy_(xs.view(torch.uint8))
    a = st.stamp_fp8_linear(x, odd, w, ws, out_dtype=torch.float32)
    assert torch.equal(a, st.stamp_fp8_linear(x, xs, w, ws, out_dtype=torch.float32))


@pytest.mark.parametrize("M", [1, 60, 600])
def test_results_repeat_bit_for_bit_on_other_streams(st, M):
    import torch
    x, xs = codes_of(st, M, 4096, seed=3)
    w, ws = weights_of(st, (520, 4096), seed=3)
    first = st.stamp_fp8_linear(x, xs, w, ws, out_dtype=torch.float32)
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(other):
        again = [st.stamp_fp8_linear(x, xs, w, ws, out_dtype=torch.float32) for _ in range(4)]
    torch.cuda.current_stream().wait_stream(other)
    assert all(torch.equal(first, a) for a in again)


def test_the_chain_of_an_expert_layer_can_be_captured(st):
    import torch
    x = activations(24, 512, torch.bfloat16, seed=4).clamp_(-8, 8)
    rows = torch.arange(24, dtype=torch.int32, device="cuda")
    offsets = torch.tensor([0, 3, 3, 20, 24], dtype=torch.int32, device="cuda")
    up, up_s = weights_of(st, (4, 2 * 256, 512), seed=1)
    down, down_s = weights_of(st, (4, 512, 256), seed=2)

    def layer():
        c, s = st.stamp_fp8_quantize(x, rows=rows)
        h = st.stamp_fp8_linear_grouped(c, s, offsets, up, up_s)
        c, s = st.stamp_fp8_gated_quantize(h)
        return st.stamp_fp8_linear_grouped(c, s, offsets, down, down_s, out_dtype=torch.float32)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        layer()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = layer()
    x.copy_(activations(24, 512, torch.bfloat16, seed=5).clamp_(-8, 8))
    graph.replay()
    assert torch.equal(y, layer())
    assert st.stamp_last_device_status() == 0


def test_offsets_past_32_bits(st):
    """Activations of more than 2^31 codes: the last rows are right."""
    import torch
    K, M = 4096, (1 << 31) // 4096 + 300
    x = torch.zeros(M, K, dtype=torch.bfloat16, device="cuda")
    tail = activations(300, K, torch.bfloat16, seed=6)
    x[-300:] = tail
    c, s = st.stamp_fp8_quantize(x)
    del x
    want = st.stamp_fp8_quantize(tail)
    assert torch.equal(c[-300:].view(torch.uint8), want[0].view(torch.uint8)) and torch.equal(s[-300:].view(torch.uint8), want[1].view(torch.uint8))
    w, ws = weights_of(st, (40, K), seed=6)
    y = st.stamp_fp8_linear(c, s, w, ws, out_dtype=torch.float32)
    check_product(y[-300:], values(*want), values(w, ws, True))
    assert bool((y[:1000] == 0).all())


def load_example():
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "fp8_expert_layer.py")
    spec = importlib.util.spec_from_file_location("fp8_expert_layer", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    return example


@pytest.mark.parametrize("tokens", [1, 300])
def test_the_example_layer_against_the_plain_chain(st, tokens):
    """The calls in the order an expert layer makes them, against the same chain in 64 bits.  The first product is rounded
    to bf16: its fp32 error, K 2^-23 sum |terms| at most (K = 400, the sum about ten times the result: 5e-4), moves at most
    5e-4 / 2^-8 = 12 % of the values by one bf16 step, and one in sixteen of those moves a code by one step of 2^-3:
    sqrt(0.12 / 16) 2^-3 = 1.1e-2 of the hidden values' norm, and as much of the output's, is the most that can be left."""
    import torch
    example = load_example()
    layer = example.ExpertLayer(400, 640, 6, 2)
    x = torch.randn(tokens, 400, generator=torch.Generator(device="cuda").manual_seed(3), device="cuda").bfloat16()
    got = layer(x).double().cpu().numpy()
    rows, place, offsets, share = layer.route(x)
    ends = offsets.tolist()
    c, s = plain_quantize(x.double().cpu().numpy()[rows.cpu().numpy()])
    xv = c * np.repeat(s, BLOCK, axis=1)[:, :400]
    up, down = values(layer.up_codes, layer.up_scale, True), values(layer.down_codes, layer.down_scale, True)
    y = np.zeros((len(xv), 400))
    for e in range(6):
        run = slice(ends[e], ends[e + 1])
        h = torch.from_numpy(xv[run] @ up[e].T).to(torch.bfloat16).double().numpy()
        h = h[:, :640] / (1 + np.exp(-h[:, :640])) * h[:, 640:]
        if len(h):
            c, s = plain_quantize(h)
            y[run] = (c * np.repeat(s, BLOCK, axis=1)[:, :640]) @ down[e].T
    want = (y[place.cpu().numpy()].reshape(tokens, 2, 400) * share.double().cpu().numpy()[:, :, None]).sum(axis=1)
    # (rounding the output to bf16: 2^-8 of a value at most, less than 2^-9 of the norm)
    assert np.linalg.norm(got - want) <= (1.1e-2 + 2.0 ** -9) * np.linalg.norm(want)


def test_the_example_runs():
    r = load_example().main(["--tokens", "200", "--features", "272", "--hidden", "256", "--experts", "4", "--top", "2", "--steps", "2"])
    assert np.isfinite(r["prompt_error"]) and len(r["step_errors"]) == 2


# ------------------------------------------------------------------------------------------ refusals
def test_arguments_are_checked(st):
    import torch
    x, xs = codes_of(st, 8, 256, seed=1)
    w, ws = weights_of(st, (3, 40, 256), seed=1)
    offsets = torch.tensor([0, 2, 4, 8], dtype=torch.int32, device="cuda")
    for bad in (lambda: st.stamp_fp8_linear(x, xs[:, :1].contiguous(), w[0], ws[0]),        # scales of another length
                lambda: st.stamp_fp8_linear(x.view(torch.uint8), xs, w[0], ws[0]),          # another type
                lambda: st.stamp_fp8_linear(x[:, :128], xs[:, :1], w[0], ws[0]),            # not dense, another K
                lambda: st.stamp_fp8_linear(x.cpu(), xs, w[0], ws[0]),
                lambda: st.stamp_fp8_linear(x, xs, w[0], ws[0], out_dtype=torch.float16),
                lambda: st.stamp_fp8_linear(x, xs, w[0], ws[0], bias=torch.zeros(40, dtype=torch.bfloat16, device="cuda")),
                lambda: st.stamp_fp8_linear(x, xs, w[0], ws[0], out=torch.empty(8, 41, device="cuda")),
                lambda: st.stamp_fp8_linear_grouped(x, xs, offsets[:-1], w, ws),
                lambda: st.stamp_fp8_linear_grouped(x, xs, offsets.long(), w, ws),
                lambda: st.stamp_fp8_quantize(torch.zeros(4, 256, dtype=torch.float16, device="cuda")),
                lambda: st.stamp_fp8_quantize(torch.zeros(4, 256, device="cuda"), rows=torch.zeros(4, dtype=torch.int64, device="cuda")),
                lambda: st.stamp_fp8_gated_quantize(torch.zeros(4, 257, device="cuda")),
                lambda: st.stamp_fp8_quantize_weights(torch.zeros(256, device="cuda"))):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: st.stamp_fp8_quantize(torch.zeros(4, 120, device="cuda")),          # K not a multiple of 16
                lambda: st.stamp_fp8_gated_quantize(torch.zeros(4, 2 * 24, device="cuda")),
                lambda: st.stamp_fp8_quantize_weights(torch.zeros(4, 24, device="cuda"))):
        with pytest.raises(st.StampError) as e:
            bad()
        assert e.value.status == 2
    assert st.stamp_last_device_status() == 0
