"""Rows so long that the block-scaled kernels' indices of features would not fit 32 bits are refused on the host (no GPU needed)."""
import pytest

from .test_fp8_abi import UNSUPPORTED, gated, grouped, linear, quantize, st, weights  # noqa: F401

LAST = (1 << 31) - 16      # the longest multiple of 16 that an int holds
MOST = (1 << 31) - 4096    # the longest row that is taken


@pytest.mark.parametrize("K", [LAST, (1 << 31) - 128, MOST + 16])
@pytest.mark.parametrize("call", [quantize, gated, weights, linear, grouped])
def test_longest_rows(st, call, K):  # noqa: F811
    sizes = {quantize: dict(K=K, ldx=K + 16, T=1, M=1), gated: dict(F=K, ldx=2 * K + 64, M=1)}.get(call, dict(K=K))
    assert call(st, **sizes) == UNSUPPORTED
    assert st.stamp_last_launch_count() == 0


def test_plan_of_the_longest_rows(st):  # noqa: F811
    for K in (LAST, MOST + 16):
        with pytest.raises(st.StampError) as e:
            st.stamp_debug_fp8_plan(4, 64, K)
        assert e.value.status == UNSUPPORTED
    assert st.stamp_debug_fp8_plan(4, 64, MOST)[1] >= 16
