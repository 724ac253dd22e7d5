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
