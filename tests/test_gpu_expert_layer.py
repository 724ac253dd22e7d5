"""The whole expert layer for a few tokens against plain statements in 64 bits.

Tolerances, derived before the first run.  Activations are taken as they are, as sums of e4m3 terms with a power-of-two scale
for each block of 128: the first term is off by at most 2^-4 of the value it stands for, every further one by 2^-5 of what was
left, and none by less than 2^-10 of its own scale, which is below 2^-18 of the block's largest value for the first and falls
as the terms do.  bf16 tokens take two terms, which hold their 8 significant bits; fp32 tokens four, 2^-19 of the value; the hidden
values three (bf16 output, 2^-14) or four (fp32 output, 2^-19).  Against the block's largest value: eps_x = 2^-20 for bf16 tokens
(what two terms cannot hold), 2^-18 for fp32 ones, eps_h = 2^-13 and 2^-18.
  gate, up  d = K 2^-23 sum |x w| + eps_x sum |blockmax w| + 2^-24 |value|   (products exact, sums in fp32 on the tensor cores)
  hidden    silu's slope is at most 1.1: dh = 1.1 dg (|u| + du) + |silu(g)| du + 2^-20 |h|
  output    over the token's rows: share (F 2^-23 sum |h w| + eps_h sum |blockmax w| + sum dh |w|), 2^-22 of every term for the
            sums around them, and half the distance of two neighbours of the output type."""
import numpy as np
import pytest

from .test_gpu_fp8 import BLOCK, st, values, weights_of  # noqa: F401

pytestmark = pytest.mark.gpu


def largest_in_block(a):
    """Each value replaced by the largest magnitude of its block of 128."""
    m, k = a.shape
    nb = -(-k // BLOCK)
    p = np.pad(np.abs(a), ((0, 0), (0, nb * BLOCK - k))).reshape(m, nb, BLOCK).max(axis=2)
    return np.repeat(p, BLOCK, axis=1)[:, :k]


def plain_layer(x, rows, share, offsets, up, down, up_bias, down_bias, residual, T, eps_x, eps_h):
    """Values in 64 bits and how far the kernels may be off, before the output's rounding."""
    N, F = down.shape[1:]
    want = np.zeros((T, N)) if residual is None else residual.copy()
    off = 2.0 ** -23 * np.abs(want)
    for e in range(len(up)):
        for m in range(offsets[e], offsets[e + 1]):
            t = rows[m]
            if t < 0 or t >= T:
                continue
            v = x[t:t + 1]
            z, d = v @ up[e].T, v.shape[1] * 2.0 ** -23 * (np.abs(v) @ np.abs(up[e]).T) + eps_x * (largest_in_block(v) @ np.abs(up[e]).T)
            if up_bias is not None:
                z = z + up_bias[e]
            d = d + 2.0 ** -24 * np.abs(z)
            g, u, dg, du = z[:, :F], z[:, F:], d[:, :F], d[:, F:]
            silu = g * np.exp(-np.logaddexp(0.0, -g))
            h, dh = silu * u, 1.1 * dg * (np.abs(u) + du) + np.abs(silu) * du + 2.0 ** -20 * np.abs(silu * u)
            w = np.abs(down[e]).T
            y = h @ down[e].T
            dy = F * 2.0 ** -23 * (np.abs(h) @ w) + eps_h * (largest_in_block(h) @ w) + dh @ w
            if down_bias is not None:
                y = y + down_bias[e]
            want[t] += share[m] * y[0]
            off[t] += abs(share[m]) * (dy[0] + 2.0 ** -22 * (np.abs(h) @ w)[0] + 2.0 ** -22 * np.abs(y[0]))
    return want, off


def check(y, want, off):
    bits = 8 if str(y.dtype) == "torch.bfloat16" else 24
    bound = off + 2.0 ** (np.floor(np.log2(np.abs(want) + off + 1e-300)) - bits)
    got = y.double().cpu().numpy()
    assert got.shape == want.shape
    bad = ~(np.abs(got - want) <= bound)
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:5].tolist(), float(np.max(np.abs(got - want) / bound)))


def routing(counts, T, seed=0, spare=0):
    """Rows in expert order for runs of these lengths: any tokens (different ones inside a run where there are enough)."""
    rng = np.random.default_rng(seed)
    rows = np.concatenate([rng.permutation(T)[:c] if c <= T else rng.integers(0, T, c) for c in counts] + [rng.integers(0, T, spare)])
    offsets = np.concatenate([[0], np.cumsum(counts)])
    return rows.astype(np.int32), rng.uniform(0.05, 1.0, len(rows)).astype(np.float32), offsets.astype(np.int32)


class Layer:
    def __init__(self, st, E, K, F, N, seed=0, bias=False):  # noqa: F811
        import torch
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.up, self.up_s = st.stamp_fp8_quantize_weights(torch.randn(E, 2 * F, K, generator=g, device="cuda") * 1.5 * K ** -0.5)
        w = torch.randn(E, N, F, generator=g, device="cuda") * F ** -0.5
        # blocks of different size, so that a scale taken from a neighbouring block shows
        w *= torch.exp2(torch.randint(-3, 4, (E, -(-N // 128), -(-F // 128)), generator=g, device="cuda").float()).repeat_interleave(128, 1)[:, :N].repeat_interleave(128, 2)[:, :, :F]
        self.down, self.down_s = st.stamp_fp8_quantize_weights(w)
        self.up_bias = torch.randn(E, 2 * F, generator=g, device="cuda") if bias else None
        self.down_bias = torch.randn(E, N, generator=g, device="cuda") if bias else None
        self.shape = E, K, F, N

    def plain(self, x, rows, share, offsets, residual, out_bf16, T):
        f64 = lambda t: None if t is None else t.double().cpu().numpy()  # noqa: E731
        return plain_layer(f64(x), rows, share, offsets, values(self.up, self.up_s, True), values(self.down, self.down_s, True), f64(self.up_bias),
                           f64(self.down_bias), f64(residual), T, 2.0 ** -20 if str(x.dtype) == "torch.bfloat16" else 2.0 ** -18,
                           2.0 ** -13 if out_bf16 else 2.0 ** -18)

    def __call__(self, st, x, rows, share, offsets, **more):  # noqa: F811
        import torch
        on = lambda a: torch.from_numpy(a).cuda()  # noqa: E731
        return st.stamp_fp8_expert_layer(x, on(rows), on(share), on(offsets), self.up, self.up_s, self.down, self.down_s, up_bias=self.up_bias,
                                         down_bias=self.down_bias, **more)


def tokens(T, K, dtype, seed=0):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(T, K, generator=g, device="cuda")
    x *= torch.where(torch.rand(K, generator=g, device="cuda") < 0.02, 20.0, 1.0)
    x *= torch.exp2(torch.randint(-2, 3, (T, 1), generator=g, device="cuda").float())
    return x.to(getattr(torch, dtype))


# tokens, rows of each expert, K, F, N
CASES = {
    "one token, one expert": (1, [1], 16, 16, 1),
    "one token": (1, [0, 1, 0, 1, 0, 0, 1, 1], 512, 256, 512),
    "short blocks": (3, [2, 0, 3, 1], 400, 272, 130),
    "hidden channels that end inside a block": (5, [5, 1, 0, 2, 3], 144, 208, 257),
    "a long sum": (2, [1, 2, 0, 1], 4096, 1040, 384),
    "many hidden channels": (2, [2, 1], 128, 4096, 128),
    "a batch": (24, [3, 0, 9, 1, 24, 7, 0, 4], 640, 384, 640),
    "all tokens to one expert": (64, [0, 64, 0], 256, 256, 264),
    "many rows for each": (64, [64, 40, 33, 17, 16, 15], 384, 640, 384),
    "more rows than tokens": (7, [20, 50, 3], 128, 128, 128),
    "many experts": (16, [1, 0, 0, 2] * 40, 128, 144, 136),
    "few features, many hidden channels": (9, [3, 0, 4, 1, 2], 256, 4096, 520),
    "many output channels": (9, [1] * 28, 128, 512, 3968),
    "no rows": (4, [0, 0, 0], 128, 128, 128),
}


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("name", list(CASES))
def test_against_the_definition(st, name, dtype):  # noqa: F811
    import torch
    T, counts, K, F, N = CASES[name]
    layer = Layer(st, len(counts), K, F, N, seed=len(name), bias=len(name) % 2 == 0)
    rows, share, offsets = routing(counts, T, seed=T)
    x = tokens(T, K, dtype, seed=T)
    for out in (torch.bfloat16, torch.float32):
        for residual in (None, torch.randn(T, N, device="cuda").bfloat16()):
            y = layer(st, x, rows, share, offsets, residual=residual, out_dtype=out)
            assert y.dtype == out and st.stamp_last_launch_count() <= 2
            check(y, *layer.plain(x, rows, share, offsets, residual, out == torch.bfloat16, T))
    assert st.stamp_last_device_status() == 0


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("counts", [[2] * 1024, [0, 2048, 0], [1] * 64 + [0] * 955 + [300, 1, 0, 5, 6]], ids=["two for each", "all to one", "uneven"])
def test_the_largest_tables(st, counts, dtype):  # noqa: F811
    """As many tokens, rows and experts as the call takes; every token comes up many times, in one run too."""
    import torch
    T, K, F, N = 64, 32, 48, 72
    layer = Layer(st, len(counts), K, F, N, seed=7)
    rows, share, offsets = routing(counts, T, seed=7, spare=2048 - sum(counts))
    x, residual = tokens(T, K, dtype), tokens(T, N, dtype, seed=8)
    for out in (torch.bfloat16, torch.float32):
        y = layer(st, x, rows, share, offsets, residual=residual, out_dtype=out)
        want, off = layer.plain(x, rows, share, offsets, residual, out is torch.bfloat16, T)
        # (a token's many rows are added one by one: each addition is rounded once more)
        check(y, want, off + 2048 * 2.0 ** -24 * np.abs(want))
    assert st.stamp_last_device_status() == 0


def test_typical_errors_are_far_below_the_worst_case(st):  # noqa: F811
    """The bounds above grow with the lengths of the sums.  Errors of either sign grow with their roots: as a share of the
    output's norm an fp32 layer stays below 2e-5 and a bf16 one within the 2^-9 of its own rounding."""
    import torch
    layer = Layer(st, 8, 1152, 768, 1152, seed=3)
    rows, share, offsets = routing([4, 1, 0, 7, 16, 2, 0, 3], 16, seed=5)
    for dtype, out, most in (("float32", torch.float32, 2e-5), ("bfloat16", torch.bfloat16, 2.0 ** -9)):
        x = tokens(16, 1152, dtype, seed=6)
        want = layer.plain(x, rows, share, offsets, None, False, 16)[0]
        y = layer(st, x, rows, share, offsets, out_dtype=out).double().cpu().numpy()
        assert np.linalg.norm(y - want) <= most * np.linalg.norm(want)


@pytest.mark.parametrize("T,counts,K,F,N", [(1, [1, 0, 1], 256, 128, 128), (3, [3, 0, 1, 2], 1152, 384, 257), (64, [64, 1, 33, 0, 16], 512, 208, 520),
                                            (20, [1, 0, 4, 2] * 16, 272, 640, 1152), (40, [40, 31], 4096, 256, 136)])
def test_integers_come_out_exact(st, T, counts, K, F, N):  # noqa: F811
    """Gates of 128 from their bias alone leave silu(g) = 128 exactly; ups are sums of small integers, shares powers of two: every
    value fits the terms and every sum is exact in fp32, so that the output equals the definition bit for bit."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(T + K)
    E = len(counts)

    def integers(low, high, *shape):
        return torch.randint(low, high, shape, generator=g, device="cuda")

    def e8m0(exponent):
        return (exponent + 127).to(torch.uint8).view(torch.float8_e8m0fnu)

    def spread(exponent, rows, columns):
        return torch.exp2(exponent.double()).repeat_interleave(BLOCK, 1)[:, :rows].repeat_interleave(BLOCK, 2)[:, :, :columns]

    up, down = torch.zeros(E, 2 * F, K, device="cuda"), integers(-2, 3, E, N, F).float()
    # eight features of each up channel count, wherever they lie: |u| <= 8 * 2 * 2 * 2 = 64, multiples of 1/2
    at = torch.rand(E, F, K, generator=g, device="cuda").topk(8, dim=2).indices
    up[:, F:].scatter_(2, at, integers(-2, 3, E, F, 8).float())
    eu, ed = integers(-1, 2, E, -(-2 * F // BLOCK), -(-K // BLOCK)), integers(-1, 2, E, -(-N // BLOCK), -(-F // BLOCK))
    up_bias, down_bias = torch.zeros(E, 2 * F, device="cuda"), integers(-9, 10, E, N).float()
    up_bias[:, :F] = 128.0
    up_bias[:, F:] = integers(-3, 4, E, F).float()
    x = integers(-2, 3, T, K).float()
    rows, _, offsets = routing(counts, T, seed=T)
    share = np.exp2(np.random.default_rng(T).integers(-1, 2, len(rows))).astype(np.float32)
    u64, d64 = up.double() * spread(eu, 2 * F, K), down.double() * spread(ed, N, F)
    residual = integers(-20, 21, T, N).float()
    want = residual.double()
    for e in range(E):
        for m in range(offsets[e], offsets[e + 1]):
            z = u64[e] @ x[rows[m]].double() + up_bias[e].double()
            want[rows[m]] += float(share[m]) * (d64[e] @ (z[:F] * z[F:]) + down_bias[e].double())
    assert float(want.abs().max()) < 2 ** 22
    args = [torch.from_numpy(a).cuda() for a in (rows, share, offsets)]
    weights = (up.to(torch.float8_e4m3fn), e8m0(eu), down.to(torch.float8_e4m3fn), e8m0(ed))
    for dtype in (torch.bfloat16, torch.float32):
        for _ in range(3):
            y = torch.full((T, N), float("nan"), device="cuda")
            st.stamp_fp8_expert_layer(x.to(dtype), *args, *weights, up_bias=up_bias, down_bias=down_bias, residual=residual, out=y)
            wrong = y != want.float()
            assert not bool(wrong.any()), (dtype, int(wrong.sum()), torch.nonzero(wrong)[:4].tolist())
    assert st.stamp_last_device_status() == 0


@pytest.mark.parametrize("T,counts,K,F,N", [(1, [1, 0, 1], 34048, 128, 128), (3, [3, 0, 1, 2], 128, 8448, 257), (20, [1, 0, 4, 20] * 16, 8464, 144, 136),
                                            (33, [33, 40], 4224, 4240, 136), (13, [13, 2, 5, 0, 1, 3], 12304, 784, 264)])
def test_integers_come_out_exact_in_several_parts(st, T, counts, K, F, N):  # noqa: F811
    """Sums of more than 4096 features, gates' and ups' as well as the way down's, in clusters and in one CTA."""
    test_integers_come_out_exact(st, T, counts, K, F, N)


@pytest.mark.parametrize("T,counts,K,F,N,down", [(16, [1] * 32, 272, 640, 1664, 10), (20, [1, 0, 4, 2] * 16, 144, 784, 2560, 10), (9, [2, 1, 3] * 12, 128, 656, 3200, 9),
                                                 (13, [1] * 40, 128, 528, 3584, 8), (40, [40, 9, 33, 17] * 3, 128, 1296, 1536, 16)])
def test_integers_come_out_exact_in_clusters_of_every_size(st, T, counts, K, F, N, down):  # noqa: F811
    assert st.stamp_debug_expert_plan(T, sum(counts), len(counts), K, F, N)[1] == down
    test_integers_come_out_exact(st, T, counts, K, F, N)


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("T,counts,K,F,N", [(1, [1, 0, 1], 1152, 2048, 1152), (13, [2, 0, 13, 1, 0, 5], 400, 272, 257), (64, [64, 33, 1, 16], 512, 640, 520)])
def test_the_output_type_costs_its_own_rounding_only(st, T, counts, K, F, N, dtype):  # noqa: F811
    """A bf16 output is the fp32 output rounded once: hidden values and sums do not depend on it."""
    import torch
    layer = Layer(st, len(counts), K, F, N, seed=K, bias=True)
    rows, share, offsets = routing(counts, T, seed=T)
    x, residual = tokens(T, K, dtype, seed=1), tokens(T, N, dtype, seed=2)
    wide, narrow = (layer(st, x, rows, share, offsets, residual=residual, out_dtype=t) for t in (torch.float32, torch.bfloat16))
    assert torch.equal(narrow, wide.bfloat16())


@pytest.mark.parametrize("E,K,F", [(1, 262144, 128), (40, 65536, 16), (8, 16, 65536)], ids=["features, a cluster", "features, one CTA", "hidden channels"])
def test_long_sums_are_taken_in_parts(st, E, K, F):  # noqa: F811
    """The tensor cores cut a running sum off instead of rounding it: 4e-7 of a sum of 4096 features against 64 bits, as a share of
    the norm, and more with every further feature of the same accumulator.  The errors of parts add up like the parts
    themselves, so that it is no more than 4e-7 again for parts of 4096 and fewer, however long the sum.  Gates of 128 from their bias alone leave silu(g) = 128, bf16 tokens are held exactly, and fp32
    hidden values' four terms are off by 2^-20 at most, 2^-20 / sqrt(3) as a root mean square: 6.8e-7 altogether, below 2^-20."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(E + K)
    N = 256
    x, up, down = torch.randn(E, K, generator=g, device="cuda").bfloat16(), torch.zeros(E, 2 * F, K, device="cuda"), torch.randn(E, N, F, generator=g, device="cuda")
    up[:, F:] = torch.randn(E, F, K, generator=g, device="cuda")
    (up, up_s), (down, down_s) = st.stamp_fp8_quantize_weights(up), st.stamp_fp8_quantize_weights(down)
    up_bias = torch.zeros(E, 2 * F, device="cuda")
    up_bias[:, :F] = 128.0
    each = torch.arange(E + 1, dtype=torch.int32, device="cuda")
    y = st.stamp_fp8_expert_layer(x, each[:-1].contiguous(), torch.ones(E, device="cuda"), each, up, up_s, down, down_s, up_bias=up_bias, out_dtype=torch.float32)
    exact = lambda c, s: c.double() * s.double().repeat_interleave(BLOCK, 0)[:c.shape[0]].repeat_interleave(BLOCK, 1)[:, :c.shape[1]]  # noqa: E731
    want = torch.stack([exact(down[e], down_s[e]) @ (128 * (exact(up[e], up_s[e])[F:] @ x[e].double())) for e in range(E)])
    error = float((y.double() - want).norm() / want.norm())
    assert error <= 2.0 ** -20, error


def test_fp32_tokens_keep_their_last_bits(st):  # noqa: F811
    """A feature less its own first eight bits: 24 bits in five terms, so that what is left comes out to the hidden values' 2^-19."""
    import torch
    K, F = 256, 128
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.zeros(40, K, device="cuda")
    x[:, 3] = (1 + torch.rand(40, generator=g, device="cuda")) * torch.where(torch.rand(40, generator=g, device="cuda") < 0.5, 1.0, -1.0)
    x[:, 77] = x[:, 3].bfloat16().float()
    up = torch.zeros(1, 2 * F, K, device="cuda")
    up[0, F:, 3], up[0, F:, 77] = 1.0, -1.0
    up_bias = torch.zeros(1, 2 * F, device="cuda")
    up_bias[0, :F] = 128.0                                   # silu(128) = 128
    codes, scale = st.stamp_fp8_quantize_weights(up)
    dc, ds = st.stamp_fp8_quantize_weights(torch.eye(F, device="cuda")[None])
    rows, share, offsets = torch.arange(40, dtype=torch.int32, device="cuda"), torch.ones(40, device="cuda"), torch.tensor([0, 40], dtype=torch.int32, device="cuda")
    y = st.stamp_fp8_expert_layer(x, rows, share, offsets, codes, scale, dc, ds, up_bias=up_bias)
    want = 128 * (x[:, 3:4].double() - x[:, 77:78].double())
    assert bool(((y.double() - want).abs() <= 2.0 ** -18 * want.abs()).all())


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("T,counts,K,F,N", [(7, [2, 1, 0, 3, 2, 4, 1, 1], 4096, 1024, 512), (3, [1, 2, 3], 1024, 4096, 512), (20, [20, 7, 0, 13], 4096, 512, 264)])
def test_fp32_outputs_are_as_near_as_a_product_in_fp32(st, T, counts, K, F, N, dtype):  # noqa: F811
    """As a share of the norm.  Sums of 2048 features are off by 2e-7 (half of what those of 4096 are), gates and ups both count, the
    hidden values' terms are off by 2^-20 / sqrt(3), the way down's sums by 2e-7 again: 6.5e-7 altogether, below 2^-20."""
    import torch
    layer = Layer(st, len(counts), K, F, N, seed=K + F)
    rows, share, offsets = routing(counts, T, seed=T)
    x = torch.randn(T, K, generator=torch.Generator(device="cuda").manual_seed(T), device="cuda").to(getattr(torch, dtype))
    y = layer(st, x, rows, share, offsets, out_dtype=torch.float32).double().cpu().numpy()
    want = layer.plain(x, rows, share, offsets, None, False, T)[0]
    error = np.linalg.norm(y - want) / np.linalg.norm(want)
    assert error <= 2.0 ** -20, error


def test_values_far_below_their_block_are_kept(st):  # noqa: F811
    """One large value in a block leaves the others 2^-20 of it: they still count to within 2^-20 of the large one."""
    import torch
    K, F = 256, 128
    up = torch.zeros(1, 2 * F, K, device="cuda")
    up[0, F:, 5] = 1.0                                       # the up channels see a small feature only
    up_bias = torch.zeros(1, 2 * F, device="cuda")
    up_bias[0, :F] = 128.0
    down = torch.eye(F, device="cuda")[None]
    codes, scale = st.stamp_fp8_quantize_weights(up)
    dc, ds = st.stamp_fp8_quantize_weights(down)
    rows, share, offsets = (torch.tensor(a, device="cuda", dtype=d) for a, d in (([0], torch.int32), ([1.0], torch.float32), ([0, 1], torch.int32)))
    for dtype in (torch.bfloat16, torch.float32):
        for exponent in range(0, 30, 3):
            x = torch.zeros(1, K, device="cuda", dtype=dtype)
            x[0, 3], x[0, 5] = 1.0, 1.37 * 2.0 ** -exponent
            y = st.stamp_fp8_expert_layer(x, rows, share, offsets, codes, scale, dc, ds, up_bias=up_bias, out_dtype=torch.float32)
            assert float((y.double() / 128 - x[0, 5].double()).abs().max()) <= 2.0 ** -20 + 2.0 ** -18 * float(x[0, 5])


@pytest.mark.parametrize("T", [3, 40])
def test_what_is_not_finite_stays_with_its_tokens(st, T):  # noqa: F811
    import torch
    layer = Layer(st, 4, 256, 256, 256, seed=1)
    rows, share, offsets = routing([T, 2, 0, 1], T, seed=1)
    x = tokens(T, 256, "bfloat16")
    clean = layer(st, x, rows, share, offsets)
    for value in (float("inf"), float("-inf"), float("nan")):
        bad = x.clone()
        bad[1, 200] = value
        y = layer(st, bad, rows, share, offsets)
        others = [t for t in range(T) if t != 1]
        assert bool(torch.isnan(y[1]).all()) and torch.equal(y[others], clean[others])
    # weights of an expert that are NaN: its own tokens only
    layer.down_s.view(torch.uint8)[1] = 255
    hit = sorted(set(rows[offsets[1]:offsets[2]].tolist()))
    y = layer(st, x, rows, share, offsets)
    others = [t for t in range(T) if t not in hit]
    assert bool(torch.isnan(y[hit]).all()) and torch.equal(y[others], clean[others])


def test_unused_rows_and_tokens_without_any(st):  # noqa: F811
    import torch
    layer = Layer(st, 3, 128, 128, 128, seed=2)
    rows, share, offsets = routing([2, 0, 1], 6, seed=2, spare=9)
    x, residual = tokens(6, 128, "bfloat16"), torch.randn(6, 128, device="cuda").bfloat16()
    share[3:] = float("nan")
    x_used = sorted(set(rows[:3].tolist()))
    y = layer(st, x, rows, share, offsets, residual=residual)
    check(y, *layer.plain(x, rows[:3], share[:3], offsets, residual, True, 6))
    for t in range(6):
        if t not in x_used:
            assert torch.equal(y[t], residual[t])
    assert bool((layer(st, x, rows, share, offsets)[[t for t in range(6) if t not in x_used]] == 0).all())


@pytest.mark.parametrize("bad", [[0, 5, 4, 9], [1, 2, 3, 9], [0, 2, 4, 10], [0, -1, 4, 9], [0, 2, 1 << 30, 9]])
def test_offsets_out_of_order_write_nothing_and_are_reported(st, bad):  # noqa: F811
    import torch
    layer = Layer(st, 3, 128, 128, 128, seed=2)
    rows, share, _ = routing([3, 3, 3], 5, seed=3)
    y = torch.full((5, 128), 7.0, device="cuda")
    layer(st, tokens(5, 128, "bfloat16"), rows, share, np.array(bad, dtype=np.int32), out=y)
    assert st.stamp_last_device_status() == 1 and st.stamp_last_device_status() == 0
    assert bool((y == 7).all())


def test_tokens_out_of_range_add_nothing_and_are_reported(st):  # noqa: F811
    layer = Layer(st, 3, 128, 128, 128, seed=2)
    rows, share, offsets = routing([3, 1, 5], 5, seed=3)
    rows[[0, 4, 6]] = -1, 5, 1 << 30
    x = tokens(5, 128, "bfloat16")
    y = layer(st, x, rows, share, offsets)
    assert st.stamp_last_device_status() == 1 and st.stamp_last_device_status() == 0
    check(y, *layer.plain(x, rows, share, offsets, None, True, 5))


def test_rows_of_a_wider_matrix_an_output_off_the_alignment_and_in_place(st):  # noqa: F811
    import torch
    layer = Layer(st, 4, 144, 128, 130, seed=4)
    rows, share, offsets = routing([2, 0, 3, 1], 5, seed=4)
    for dtype in ("bfloat16", "float32"):
        wide = tokens(5, 144 + 32, dtype)
        x = wide[:, 16:160]
        want = layer(st, x.contiguous(), rows, share, offsets)
        assert torch.equal(layer(st, x, rows, share, offsets), want)
        room = torch.full((5 * 130 + 65,), 7.0, dtype=x.dtype, device="cuda")
        y = layer(st, x, rows, share, offsets, out=room[33:33 + 650].view(5, 130))
        assert torch.equal(y, want) and bool((room[:33] == 7).all()) and bool((room[-32:] == 7).all())
        r = torch.randn(5, 133, device="cuda").to(x.dtype)[:, 1:131]
        want = layer(st, x, rows, share, offsets, residual=r)
        r = r.contiguous()
        layer(st, x, rows, share, offsets, residual=r, out=r)
        assert torch.equal(r, want)


@pytest.mark.parametrize("T", [1, 30])
def test_results_repeat_on_other_streams_and_with_given_scratch(st, T):  # noqa: F811
    import torch
    layer = Layer(st, 8, 512, 512, 512, seed=5)
    rows, share, offsets = routing([1, 0, min(T, 9), 1, T, 0, 1, 1], T, seed=5)
    x = tokens(T, 512, "bfloat16")
    first = layer(st, x, rows, share, offsets, out_dtype=torch.float32)
    ws = torch.full((st.stamp_fp8_expert_workspace_bytes(len(rows), 512),), 0xFF, dtype=torch.uint8, device="cuda")     # (NaN to begin with)
    streams = [torch.cuda.Stream() for _ in range(2)]
    again = []
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):      # two streams at once, each with scratch of its own
            again += [layer(st, x, rows, share, offsets, out_dtype=torch.float32) for _ in range(4)]
    for s in streams:
        torch.cuda.current_stream().wait_stream(s)
    again += [layer(st, x, rows, share, offsets, out_dtype=torch.float32, ws=ws) for _ in range(2)]
    assert all(torch.equal(first, a) for a in again)


def test_a_decode_step_from_the_logits_on(st):  # noqa: F811
    """Router's choice and layer, as a decode step runs them: captured, replayed on new inputs, and against the chain of the
    quantized calls that a prompt takes, which differ by the tokens' and hidden values' rounding to e4m3 (2^-4 of a value at
    most, 2^-5.3 on average of both: 4 % of the output's norm)."""
    import torch
    T, E, K, F, top = 12, 16, 512, 384, 4
    layer = Layer(st, E, K, F, K, seed=6)
    router = torch.randn(K, E, device="cuda") * K ** -0.5
    x = tokens(T, K, "bfloat16")

    def step():
        _, _, rows, _, offsets, row_share = st.stamp_expert_route(x.float() @ router, top)
        return st.stamp_fp8_expert_layer(x, rows, row_share, offsets, layer.up, layer.up_s, layer.down, layer.down_s, residual=x)

    def prompt():
        _, share, rows, place, offsets, _ = st.stamp_expert_route(x.float() @ router, top)
        c, s = st.stamp_fp8_quantize(x, rows=rows)
        h = st.stamp_fp8_linear_grouped(c, s, offsets, layer.up, layer.up_s)
        c, s = st.stamp_fp8_gated_quantize(h)
        y = st.stamp_fp8_linear_grouped(c, s, offsets, layer.down, layer.down_s)
        return st.stamp_expert_combine(y, place, share, residual=x)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
        prompt()
    torch.cuda.current_stream().wait_stream(side)
    graphs, outs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()], []
    for graph, form in zip(graphs, (step, prompt)):
        with torch.cuda.graph(graph):
            outs.append(form())
    x.copy_(tokens(T, K, "bfloat16", seed=9))
    for _ in range(2):
        for graph in graphs:
            graph.replay()
    for out, form in zip(outs, (step, prompt)):
        assert torch.equal(out, form())
    a, b, r = (t.double().cpu().numpy() for t in (outs[0], outs[1], x))
    assert np.linalg.norm(a - b) <= 0.08 * np.linalg.norm(b - r)
    assert st.stamp_last_device_status() == 0


def test_the_example_decodes(st):  # noqa: F811
    """The example's step of a few tokens against the definition of the layer on its quantized weights."""
    import importlib.util
    import os

    import torch
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "fp8_expert_layer.py")
    spec = importlib.util.spec_from_file_location("fp8_expert_layer", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    layer = example.ExpertLayer(272, 384, 6, 2)
    x, residual = tokens(7, 272, "bfloat16"), tokens(7, 272, "bfloat16", seed=4)
    y = layer.decode(x, residual)
    rows, place, offsets, share = (t.cpu().numpy() for t in layer.route(x))
    row_share = np.empty(14, dtype=np.float32)
    row_share[place.reshape(-1)] = share.reshape(-1)
    up, down = (values(c, s, True) for c, s in ((layer.up_codes, layer.up_scale), (layer.down_codes, layer.down_scale)))
    check(y, *plain_layer(x.double().cpu().numpy(), rows, row_share, offsets, up, down, None, None, residual.double().cpu().numpy(), 7, 2.0 ** -20, 2.0 ** -13))


@pytest.mark.parametrize("T", [1, 5, 64])
def test_the_output_may_be_over_the_tokens(st, T):  # noqa: F811
    """A step in place: tokens, residual and output are one matrix, or the output starts inside the tokens."""
    import torch
    for dtype in (torch.bfloat16, torch.float32):
        layer = Layer(st, 6, 256, 384, 256, seed=T)
        rows, share, offsets = routing([T, 1, 0, 1, T, 0], T, seed=T)
        x = tokens(T, 256, str(dtype).split(".")[1], seed=T)
        want, alone = layer(st, x, rows, share, offsets, residual=x), layer(st, x, rows, share, offsets)
        for _ in range(4):
            y = x.clone()
            layer(st, y, rows, share, offsets, residual=y, out=y)
            assert torch.equal(y, want)
            room = torch.zeros(T * 256 + 128, dtype=dtype, device="cuda")
            room[:T * 256] = x.view(-1)
            y = room[128:].view(T, 256)
            layer(st, room[:T * 256].view(T, 256), rows, share, offsets, out=y)
            assert torch.equal(y, alone)
    assert st.stamp_last_device_status() == 0


def test_arguments_are_checked(st):  # noqa: F811
    import torch
    layer = Layer(st, 4, 128, 128, 128, seed=2)
    rows, share, offsets = (torch.from_numpy(a).cuda() for a in routing([2, 0, 3, 1], 5, seed=4))
    x = tokens(5, 128, "bfloat16")
    w = (layer.up, layer.up_s, layer.down, layer.down_s)
    call = st.stamp_fp8_expert_layer
    for bad in (lambda: call(x.half(), rows, share, offsets, *w), lambda: call(x.cpu(), rows, share, offsets, *w), lambda: call(x[0], rows, share, offsets, *w),
                lambda: call(x, rows.long(), share, offsets, *w), lambda: call(x, rows, share[:5], offsets, *w), lambda: call(x, rows, share, offsets[:4], *w),
                lambda: call(x, rows, share, offsets, layer.up[0], *w[1:]), lambda: call(x, rows, share, offsets, layer.up, layer.up_s[:, :1].contiguous(), *w[2:]),
                lambda: call(x, rows, share, offsets, *w, up_bias=torch.zeros(4, 128, device="cuda")), lambda: call(x, rows, share, offsets, *w, residual=x[:4]),
                lambda: call(x, rows, share, offsets, *w, out_dtype=torch.float16), lambda: call(x, rows, share, offsets, *w, ws=torch.empty(9)),
                lambda: call(x[:, :64], rows, share, offsets, *w)):
        with pytest.raises(ValueError):
            bad()
    many = torch.zeros(65, 128, dtype=torch.bfloat16, device="cuda")
    long_rows = torch.zeros(2049, dtype=torch.int32, device="cuda")
    for status, bad in ((2, lambda: call(many, rows, share, offsets, *w)), (2, lambda: call(x, long_rows, long_rows.float(), offsets, *w)),
                        (3, lambda: call(x, rows, share, offsets, *w, ws=torch.empty(256, dtype=torch.uint8, device="cuda"))),
                        (1, lambda: call(torch.zeros(5, 132, dtype=torch.bfloat16, device="cuda")[:, 1:129], rows, share, offsets, *w))):
        with pytest.raises(st.StampError) as e:
            bad()
        assert e.value.status == status
    assert call(x[:0], rows[:0], share[:0], offsets * 0, *w).shape == (0, 128)
    assert st.stamp_last_device_status() == 0
