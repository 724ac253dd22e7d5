"""The block-scaled products kernel by kernel: CTA pairs and single CTAs, every height of tile, sums in one accumulator, in
several, and split over a cluster.  Each test states the kernel it means and asks the library whether the sizes run it.

Codes are small integers and scales powers of two, so that every term is a multiple of 1/4 and a sum of any of them stays
below 2^24 quarters: every partial sum is exact in fp32, in whatever order and with whatever rounding, and the fp32 output has
to equal the sum in 64 bits bit for bit (the bf16 output, that sum rounded once).  Outputs start as NaN."""
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


def blocks(n):
    return -(-n // BLOCK)


class Exact:
    """Operands of a product of integers and its value in 64 bits; counts: rows of each expert, None for one matrix."""

    def __init__(self, M, K, N, counts=None, bias=False, seed=0):
        import torch
        g = torch.Generator(device="cuda").manual_seed(seed + M + K + N)
        E, kb, nb = 1 if counts is None else len(counts), blocks(K), blocks(N)

        def integers(low, high, *shape):
            return torch.randint(low, high, shape, device="cuda", generator=g)

        def e8m0(exponent):
            return (exponent + 127).to(torch.uint8).view(torch.float8_e8m0fnu)

        x, w = integers(-3, 4, M, K).float(), integers(-3, 4, E, N, K).float()
        ex, ew = integers(0, 3, M, kb), integers(-2, 1, E, nb, kb)
        self.bias = integers(-9, 10, E, N).float() if bias else None
        self.offsets = None if counts is None else torch.tensor(np.concatenate([[0], np.cumsum(counts)]), dtype=torch.int32, device="cuda")
        self.x, self.xs, self.w, self.ws = x.to(torch.float8_e4m3fn), e8m0(ex), w.to(torch.float8_e4m3fn), e8m0(ew)
        ends = [0, M] if counts is None else self.offsets.tolist()
        self.value = torch.zeros(M, N, dtype=torch.float64, device="cuda")
        xv = x.double() * torch.exp2(ex.double()).repeat_interleave(BLOCK, 1)[:, :K]
        for e in range(E):
            scale = torch.exp2(ew[e].double()).repeat_interleave(BLOCK, 1)[:, :K].repeat_interleave(BLOCK, 0)[:N]
            rows = slice(ends[e], ends[e + 1])
            self.value[rows] = xv[rows] @ (w[e].double() * scale).t() + (self.bias[e].double() if bias else 0.0)
        assert float(self.value.abs().max()) < 2 ** 22
        if counts is None:
            self.w, self.ws, self.bias = self.w[0], self.ws[0], None if self.bias is None else self.bias[0]

    def holds(self, st, dtype, repeats=1):
        import torch
        want = self.value.to(torch.float32).to(dtype)   # (exact in fp32: rounded once)
        for _ in range(repeats):
            y = torch.full(tuple(self.value.shape), float("nan"), dtype=dtype, device="cuda")
            if self.offsets is None:
                st.stamp_fp8_linear(self.x, self.xs, self.w, self.ws, bias=self.bias, out=y)
            else:
                st.stamp_fp8_linear_grouped(self.x, self.xs, self.offsets, self.w, self.ws, bias=self.bias, out=y)
            wrong = y != want                           # (true for NaN too)
            assert not bool(wrong.any()), (int(wrong.sum()), torch.nonzero(wrong)[:4].tolist())
        assert st.stamp_last_device_status() == 0


# ------------------------------------------------------------------------------------------ sums in several accumulators
# An fp32 sum of more than 4096 features takes one accumulator after the other and is added up in the output.  Sums whose
# last accumulator holds little (16, 128 and 512 features) leave the least time between one being drained and the next.
LONG = [4112, 4224, 4608, 8704, 14336]


@pytest.mark.parametrize("K", LONG)
@pytest.mark.parametrize("M,N,rows", [(1024, 4096, 256), (777, 4104, 224), (2048, 4095, 256)])
def test_pairs_add_up_long_sums(st, M, N, rows, K):
    import torch
    assert st.stamp_debug_fp8_plan(M, N, K, out_dtype=torch.float32) == (True, rows, 1)
    Exact(M, K, N, bias=True).holds(st, torch.float32, repeats=6)


@pytest.mark.parametrize("K", LONG[:4])
def test_pairs_add_up_long_sums_of_experts(st, K):
    import torch
    counts = [900, 513, 0, 1301, 1, 290]
    assert st.stamp_debug_fp8_plan(sum(counts), 2056, K, experts=len(counts), out_dtype=torch.float32) == (True, 256, 1)
    Exact(sum(counts), K, 2056, counts, bias=True).holds(st, torch.float32, repeats=6)


@pytest.mark.parametrize("M,N,K,rows", [(300, 2056, 8704, 64), (1024, 1152, 28672, 64), (448, 520, 28672, 16), (1024, 2056, 4112, 128)])
def test_single_ctas_add_up_long_sums(st, M, N, K, rows):
    import torch
    assert st.stamp_debug_fp8_plan(M, N, K, out_dtype=torch.float32) == (False, rows, 1)
    Exact(M, K, N, bias=True).holds(st, torch.float32, repeats=2)


# ------------------------------------------------------------------------------------------ every kernel, every height
@pytest.mark.parametrize("out", ["bfloat16", "float32"])
@pytest.mark.parametrize("M,N,K,rows", [(256, 6000, 8208, 128), (300, 8199, 2064, 160), (350, 8200, 2064, 192), (700, 4095, 4096, 192),
                                        (448, 8200, 2064, 224), (700, 6001, 2064, 256), (1000, 4104, 14336, 256)])
def test_pairs_of_every_height(st, M, N, K, rows, out):
    import torch
    dtype = getattr(torch, out)
    assert st.stamp_debug_fp8_plan(M, N, K, out_dtype=dtype) == (True, rows, 1)
    Exact(M, K, N, bias=True, seed=rows).holds(st, dtype)


@pytest.mark.parametrize("out", ["bfloat16", "float32"])
@pytest.mark.parametrize("M,N,K,rows,split", [
    (1, 6000, 4096, 16, 2), (17, 6000, 4096, 32, 2), (65, 4095, 4096, 64, 2), (1, 72, 4096, 16, 4), (17, 4104, 4112, 32, 4),
    (65, 2056, 4096, 64, 4), (65, 4095, 8208, 128, 4), (1, 129, 28672, 16, 8), (17, 2056, 28672, 32, 8), (40, 2047, 28672, 64, 8),
    (100, 2056, 28672, 128, 8), (1, 128, 2064, 16, 1), (65, 4096, 2064, 32, 1), (100, 6001, 2064, 64, 1), (200, 8200, 2064, 128, 1),
])
def test_single_ctas_and_clusters_of_every_height(st, M, N, K, rows, split, out):
    import torch
    dtype = getattr(torch, out)
    assert st.stamp_debug_fp8_plan(M, N, K, out_dtype=dtype) == (False, rows, split)
    Exact(M, K, N, bias=True, seed=rows + split).holds(st, dtype)


# Runs of no row, of one, of a few and of an odd number: their last tiles are copied in pieces of 32 rows.
RAGGED = {
    "pairs of 128 rows": ([907, 1, 492], 1031, 8704, (True, 128, 1)),
    "pairs of 160 rows": ([1203, 0, 897], 1032, 2064, (True, 160, 1)),
    "pairs of 192 rows": ([449, 451, 1, 0, 899, 17, 1001, 782], 520, 4224, (True, 192, 1)),
    "pairs of 224 rows": ([33, 901, 0, 2, 1777, 1488], 519, 2064, (True, 224, 1)),
    "pairs of 256 rows": ([513, 128, 1, 0, 257, 31, 1300, 770], 2056, 2064, (True, 256, 1)),
    "128 rows": ([201, 1, 98], 4095, 2064, (False, 128, 1)),
    "128 rows, four parts": ([199, 0, 101], 1032, 8704, (False, 128, 4)),
    "64 rows, four parts": ([31, 0, 59], 1031, 8704, (False, 64, 4)),
    "16 rows, two parts": ([3, 0, 7, 1, 5, 2], 1032, 4224, (False, 16, 2)),
}


@pytest.mark.parametrize("out", ["bfloat16", "float32"])
@pytest.mark.parametrize("name", list(RAGGED))
def test_runs_of_every_length(st, name, out):
    import torch
    counts, N, K, plan = RAGGED[name]
    dtype = getattr(torch, out)
    assert st.stamp_debug_fp8_plan(sum(counts), N, K, experts=len(counts), out_dtype=dtype) == plan
    Exact(sum(counts), K, N, counts, bias=True).holds(st, dtype)


@pytest.mark.parametrize("out", ["bfloat16", "float32"])
@pytest.mark.parametrize("last", [0, 1, 256, 511])
def test_pairs_write_only_the_rows_of_the_runs(st, last, out):
    """Rows behind the last run and the room around the output stay as they were, wherever the last run ends."""
    import torch
    M, N, K, guard = 1400, 4095, 2064, 4096
    dtype = getattr(torch, out)
    size = torch.empty(0, dtype=dtype).element_size()
    counts = [700, 0, 188, last]
    rows = sum(counts)
    assert st.stamp_debug_fp8_plan(M, N, K, experts=4, out_dtype=dtype)[0]
    case = Exact(rows, K, N, counts)
    # the operands reach on behind the last run; what lies there belongs to nobody (codes and scales of NaN)
    x = torch.full((M, K), 0x7F, dtype=torch.uint8, device="cuda")
    xs = torch.full((M, blocks(K)), 0xFF, dtype=torch.uint8, device="cuda")
    x[:rows], xs[:rows] = case.x.view(torch.uint8), case.xs.view(torch.uint8)
    raw = torch.full((M * N * size + 2 * guard,), 0x5A, dtype=torch.uint8, device="cuda")
    y = raw[guard:guard + M * N * size].view(dtype).view(M, N)
    st.stamp_fp8_linear_grouped(x.view(case.x.dtype), xs.view(case.xs.dtype), case.offsets, case.w, case.ws, out=y)
    assert torch.equal(y[:rows], case.value.float().to(dtype))
    assert bool((raw[:guard + rows * N * size] == 0x5A)[:guard].all()) and bool((raw[guard + rows * N * size:] == 0x5A).all())
    assert st.stamp_last_device_status() == 0


def test_pairs_refuse_offsets_out_of_order(st):
    import torch
    M, N, K = 1400, 2056, 4224
    case = Exact(M, K, N, [700, 0, 400, 300])
    assert st.stamp_debug_fp8_plan(M, N, K, experts=4, out_dtype=torch.float32)[0]
    for bad in ([0, 900, 899, 1000, 1400], [0, 1, 2, 3, 1401], [1, 2, 3, 4, 5], [0, -1, 5, 6, 7]):
        y = torch.full((M, N), 7.0, device="cuda")
        st.stamp_fp8_linear_grouped(case.x, case.xs, torch.tensor(bad, dtype=torch.int32, device="cuda"), case.w, case.ws, out=y)
        assert st.stamp_last_device_status() == 1 and st.stamp_last_device_status() == 0
        assert bool((y == 7.0).all())
    case.holds(st, torch.float32)


@pytest.mark.parametrize("out", ["bfloat16", "float32"])
def test_non_finite_rows_of_pairs_stay_alone(st, out):
    import torch
    M, N, K = 1024, 4096, 4608
    dtype = getattr(torch, out)
    assert st.stamp_debug_fp8_plan(M, N, K, out_dtype=dtype) == (True, 256, 1)
    case = Exact(M, K, N)
    bad = torch.zeros(M, dtype=torch.bool, device="cuda")
    for row, block in ((0, 0), (255, 35), (256, 33), (700, 31), (1023, 4)):
        case.xs.view(torch.uint8)[row, block] = 0xFF
        case.x.view(torch.uint8)[row, block * BLOCK:(block + 1) * BLOCK] = 0x7F
        bad[row] = True
    y = st.stamp_fp8_linear(case.x, case.xs, case.w, case.ws, out_dtype=dtype)
    assert bool(torch.isnan(y[bad]).all()) and torch.equal(y[~bad], case.value[~bad].float().to(dtype))


# ------------------------------------------------------------------------------------------ rounding, repeats, streams
@pytest.mark.parametrize("out", ["bfloat16", "float32"])
@pytest.mark.parametrize("M,N,K", [(1024, 4096, 4096), (1024, 4096, 14336), (777, 4104, 4224), (300, 2056, 14336), (17, 4096, 14336), (1, 4096, 4096)])
def test_the_sums_rounding(st, M, N, K, out):
    """An instruction adds 32 features to the running sum and is off by one unit of its last place at most, 2^-23 of it.
    The terms' signs are random, so no running sum is larger, in the mean square, than the last one: n instructions of an
    accumulator leave at most n 2^-23 of its share, p shares of like size sqrt(p) times that of the whole; the output's own
    rounding is at most 2^-9 (bf16) or p 2^-24 (fp32, the shares added up)."""
    import torch
    from .test_gpu_fp8 import activations, weights_of
    dtype = getattr(torch, out)
    x, xs = st.stamp_fp8_quantize(activations(M, K, torch.bfloat16, seed=M + K))
    w, ws = weights_of(st, (N, K), seed=K)
    y = st.stamp_fp8_linear(x, xs, w, ws, out_dtype=dtype)
    xv = x.double() * xs.double().repeat_interleave(BLOCK, 1)[:, :K]
    wv = w.double() * ws.double().repeat_interleave(BLOCK, 1)[:, :K].repeat_interleave(BLOCK, 0)[:N]
    want = xv @ wv.t()
    chunk = K if out == "bfloat16" else min(K, 4096)
    parts = -(-K // chunk)
    bound = chunk / 32 * 2.0 ** -23 * parts ** 0.5 + (2.0 ** -9 if out == "bfloat16" else parts * 2.0 ** -24)
    scale = want.norm(dim=1, keepdim=True)            # rows are of very different size
    off = float(((y.double() - want) / scale).norm() / M ** 0.5)
    assert off <= bound, (off, bound)


@pytest.mark.parametrize("out", ["bfloat16", "float32"])
@pytest.mark.parametrize("K", [2064, 4608])
def test_pairs_repeat_bit_for_bit_on_other_streams(st, K, out):
    import torch
    from .test_gpu_fp8 import codes_of, weights_of
    dtype = getattr(torch, out)
    M, N = 1500, 4104
    assert st.stamp_debug_fp8_plan(M, N, K, out_dtype=dtype)[0]
    x, xs = codes_of(st, M, K, seed=3)
    w, ws = weights_of(st, (N, K), seed=3)
    first = st.stamp_fp8_linear(x, xs, w, ws, out_dtype=dtype)
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(other):
        again = [st.stamp_fp8_linear(x, xs, w, ws, out_dtype=dtype) for _ in range(6)]
    torch.cuda.current_stream().wait_stream(other)
    assert all(torch.equal(first, a) for a in again)
    assert st.stamp_last_device_status() == 0
