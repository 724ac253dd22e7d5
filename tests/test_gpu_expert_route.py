"""The router's choice and the way back against plain statements in 64 bits.

Tolerances, derived before the first run:
  choice   comparisons of the inputs only: experts, rows, places and offsets are equal.
  shares   exp within 2 ulp of a difference that is rounded once (|d| 2^-24 relative, d <= 200 here), a sum of at most 1024
           terms that are not negative (1024 * 2^-24 at most, in practice a tree), a division: (|d| + 1024 + 8) * 2^-24.
  combine  a sum of top + 1 terms in fp32, (top + 2) * 2^-24 * sum |terms|, and half the distance of two neighbours of the
           output type."""
import numpy as np
import pytest

from .test_gpu_fp8 import st  # noqa: F401

pytestmark = pytest.mark.gpu


def plain_route(logits, top, normalize):
    """One token after the other, one choice after the other."""
    x = logits.double().cpu().numpy()
    T, E = x.shape
    chosen, share = np.zeros((T, top), dtype=np.int64), np.zeros((T, top))
    for t in range(T):
        key = np.where(np.isnan(x[t]), -np.inf, x[t])
        order = sorted(range(E), key=lambda e: (np.isnan(x[t, e]), -key[e], e))[:top]     # NaN last, then the largest, then the lowest
        chosen[t] = order
        if np.isnan(x[t]).any():
            share[t] = np.nan
        elif x[t].max() == -np.inf:
            share[t] = 0.0
        else:
            with np.errstate(invalid="ignore"):
                w = np.exp(x[t] - x[t].max())
            share[t] = w[order] / (w[order].sum() if normalize else w.sum())
    flat = chosen.reshape(-1)
    order = np.argsort(flat, kind="stable")
    place = np.empty_like(order)
    place[order] = np.arange(order.size)
    offsets = np.concatenate([[0], np.cumsum(np.bincount(flat, minlength=E))])
    return chosen, share, order // top, place.reshape(T, top), offsets, share.reshape(-1)[order]


def check_route(got, want, spread=200.0):
    chosen, share, rows, place, offsets, row_share = (t.cpu().numpy() for t in got)
    for g, w in ((chosen, want[0]), (rows, want[2]), (place, want[3]), (offsets, want[4])):
        assert g.shape == w.shape and np.array_equal(g, w)
    for g, w in ((share, want[1]), (row_share, want[5])):
        assert g.shape == w.shape and np.array_equal(np.isnan(g), np.isnan(w))
        fine = ~np.isnan(w)
        assert (np.abs(g[fine] - w[fine]) <= (spread + 1032) * 2.0 ** -24 * w[fine] + 1e-37).all()


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("T,E,top", [(1, 1, 1), (1, 64, 8), (1, 1024, 32), (2, 8, 8), (17, 60, 6), (64, 33, 4), (128, 256, 8), (129, 31, 3), (130, 256, 2),
                                     (1000, 64, 4), (4099, 16, 1), (5000, 128, 8), (700, 1000, 5), (300, 513, 32), (16384, 32, 2)])
def test_route_against_the_definition(st, T, E, top, dtype):  # noqa: F811
    import torch
    g = torch.Generator(device="cuda").manual_seed(T + E)
    x = (2 * torch.randn(T, E, generator=g, device="cuda")).to(getattr(torch, dtype))
    for normalize in (True, False):
        check_route(st.stamp_expert_route(x, top, normalize=normalize), plain_route(x, top, normalize))
    assert st.stamp_last_launch_count() == (1 if T <= 128 else 2)


@pytest.mark.parametrize("T", [5, 128, 400])
def test_equal_logits_go_to_the_lower_expert(st, T):  # noqa: F811
    import torch
    g = torch.Generator(device="cuda").manual_seed(T)
    x = torch.randint(-2, 3, (T, 72), generator=g, device="cuda").float()
    x[x == 0] *= torch.where(torch.rand(int((x == 0).sum()), generator=g, device="cuda") < 0.5, 1.0, -1.0)   # zeros of both signs are equal
    x[0] = 0.0
    x[1] = -0.0
    for dtype in (torch.float32, torch.bfloat16):
        check_route(st.stamp_expert_route(x.to(dtype), 7), plain_route(x.to(dtype), 7, True))


@pytest.mark.parametrize("T", [9, 300])
@pytest.mark.parametrize("normalize", [True, False])
def test_masked_experts_padding_and_what_is_not_finite(st, T, normalize):  # noqa: F811
    import torch
    g = torch.Generator(device="cuda").manual_seed(T)
    x = torch.randn(T, 40, generator=g, device="cuda")
    inf, low = float("inf"), torch.finfo(torch.float32).min
    x[0] = -inf                                   # padding
    x[1, 3:] = -inf                               # fewer open experts than choices
    x[2] = low                                    # masked with the type's lowest value throughout: all equal
    x[3, 5:] = low
    x[4, 7] = float("nan")
    x[5] = float("nan")
    x[6, 2:] = float("nan")
    x[7, 0], x[7, 1] = 88.0, -88.0
    for v in (x, x.bfloat16()):
        check_route(st.stamp_expert_route(v, 6, normalize=normalize), plain_route(v, 6, normalize))
    x[8, 4] = inf                                 # exp(inf - inf): the token's shares are NaN or 0, its choice is not touched
    got = st.stamp_expert_route(x, 6, normalize=normalize)
    assert np.array_equal(got[0].cpu().numpy(), plain_route(x, 6, normalize)[0])
    assert bool(torch.isnan(got[1][8, 0]))


@pytest.mark.parametrize("E", [32, 64, 128, 256, 512])
@pytest.mark.parametrize("top", [8, 11])
def test_ties_and_what_is_not_finite_where_every_lane_has_all_its_experts(st, E, top):  # noqa: F811
    import torch
    g = torch.Generator(device="cuda").manual_seed(E + top)
    x = torch.randint(-3, 1, (170, E), generator=g, device="cuda").float()
    x[x == 0] *= torch.where(torch.rand(int((x == 0).sum()), generator=g, device="cuda") < 0.5, 1.0, -1.0)
    tiny = torch.randint(-4, 5, (E,), generator=g, device="cuda").float() * 2.0 ** -130          # subnormal numbers of both types
    nan = torch.full((2,), 0x7FC00000, dtype=torch.int32, device="cuda")
    nan[1] = 0xFFC00000 - (1 << 32)
    nan = nan.view(torch.float32)                                                              # NaNs of both signs
    x[1], x[2, 3], x[3, E - 1], x[4, 1::2] = tiny, nan[0], nan[1], nan[1]
    x[5], x[5, -2:] = nan[0], -1.0
    x[6] = float("-inf")
    x[7, 2:] = float("-inf")
    x[8] = torch.finfo(torch.bfloat16).min
    for v in (x, x.bfloat16()):
        check_route(st.stamp_expert_route(v, top), plain_route(v, top, True))


def test_logits_of_a_wider_matrix_and_given_buffers(st):  # noqa: F811
    import torch
    wide = torch.randn(200, 91, device="cuda")
    x = wide[:, 3:63]
    out = (torch.full((200, 4), -7, dtype=torch.int32, device="cuda"), torch.full((200, 4), 9.0, device="cuda"), torch.full((800,), -7, dtype=torch.int32, device="cuda"),
           torch.full((200, 4), -7, dtype=torch.int32, device="cuda"), torch.full((61,), -7, dtype=torch.int32, device="cuda"), torch.full((800,), 9.0, device="cuda"))
    got = st.stamp_expert_route(x, 4, out=out)
    assert all(a.data_ptr() == b.data_ptr() for a, b in zip(got, out))
    check_route(out, plain_route(x, 4, True))


def test_no_tokens(st):  # noqa: F811
    import torch
    got = st.stamp_expert_route(torch.empty(0, 16, device="cuda"), 4)
    assert got[4].tolist() == [0] * 17 and got[2].numel() == 0
    assert st.stamp_expert_combine(torch.empty(0, 8, device="cuda"), torch.empty(0, 2, dtype=torch.int32, device="cuda"), torch.empty(0, 2, device="cuda")).shape == (0, 8)
    assert st.stamp_last_launch_count() == 0


@pytest.mark.parametrize("T", [100, 3000])
def test_route_repeats_and_can_be_captured(st, T):  # noqa: F811
    import torch
    x = torch.randn(T, 64, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        st.stamp_expert_route(x, 8)
    torch.cuda.current_stream().wait_stream(side)
    graphs, outs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()], []
    y = torch.randn(T, 64, device="cuda")
    for graph, v in zip(graphs, (x, y)):
        with torch.cuda.graph(graph):
            outs.append(st.stamp_expert_route(v, 8))
    x.copy_(torch.randn(T, 64, device="cuda"))
    for _ in range(3):
        for graph in graphs:
            graph.replay()
    for out, v in zip(outs, (x, y)):
        assert all(torch.equal(a, b) for a, b in zip(out, st.stamp_expert_route(v, 8)))


# ------------------------------------------------------------------------------------------ the way back
def check_combine(out, y, place, share, residual):
    v, p, s = y.double().cpu().numpy(), place.cpu().numpy(), share.double().cpu().numpy()
    T, top = p.shape
    want, room = np.zeros((T, v.shape[1])), np.zeros((T, v.shape[1]))
    for j in range(top):
        live = (p[:, j] >= 0) & (p[:, j] < len(v))
        term = np.where(live[:, None], v[np.where(live, p[:, j], 0)] * s[:, j:j + 1], 0.0)
        want, room = want + term, room + np.abs(term)
    if residual is not None:
        r = residual.double().cpu().numpy()
        want, room = want + r, room + np.abs(r)
    off = (top + 2) * 2.0 ** -24 * room
    bits = 8 if str(out.dtype) == "torch.bfloat16" else 24
    bound = off + 2.0 ** (np.floor(np.log2(np.abs(want) + off + 1e-300)) - bits)
    assert (np.abs(out.double().cpu().numpy() - want) <= bound).all()


@pytest.mark.parametrize("T,top,N", [(1, 1, 1), (1, 8, 2048), (40, 8, 2048), (7, 3, 130), (33, 6, 4097), (200, 4, 1152), (3, 32, 516), (1000, 5, 72), (2, 40, 24)])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_combine_against_the_definition(st, T, top, N, dtype):  # noqa: F811
    import torch
    g = torch.Generator(device="cuda").manual_seed(T + N)
    y = torch.randn(T * top, N, generator=g, device="cuda").to(getattr(torch, dtype))
    share = torch.rand(T, top, generator=g, device="cuda")
    place = torch.randperm(T * top, generator=g, device="cuda").to(torch.int32).view(T, top)
    for out in (torch.float32, torch.bfloat16):
        for residual in (None, torch.randn(T, N, device="cuda"), torch.randn(T, N + 3, device="cuda").bfloat16()[:, 1:1 + N]):
            check_combine(st.stamp_expert_combine(y, place, share, residual=residual, out_dtype=out), y, place, share, residual)
    r = torch.randn(T, N, device="cuda").bfloat16()
    before = r.clone()
    assert st.stamp_expert_combine(y, place, share, residual=r, out=r).data_ptr() == r.data_ptr()       # in place
    check_combine(r, y, place, share, before)
    assert st.stamp_last_device_status() == 0


def test_the_same_row_twice_and_places_out_of_range(st):  # noqa: F811
    import torch
    y, share = torch.randn(6, 260, device="cuda"), torch.rand(4, 3, device="cuda")
    place = torch.tensor([[0, 0, 0], [5, 1, 5], [2, 3, 4], [1, 1, 2]], dtype=torch.int32, device="cuda")
    check_combine(st.stamp_expert_combine(y, place, share, out_dtype=torch.float32), y, place, share, None)
    assert st.stamp_last_device_status() == 0
    place[1, 0], place[2, 1], place[3] = -1, 6, 1 << 30
    out = st.stamp_expert_combine(y, place, share, out_dtype=torch.float32)
    assert st.stamp_last_device_status() == 1 and st.stamp_last_device_status() == 0
    check_combine(out, y, place, share, None)
    assert bool((out[3] == 0).all())


def test_rows_past_32_bits(st):  # noqa: F811
    """More than 2^31 values to combine: the last rows are read from their own place."""
    import torch
    N, M = 4096, (1 << 31) // 4096 + 100
    y = torch.zeros(M, N, dtype=torch.bfloat16, device="cuda")
    y[-100:] = torch.randn(100, N, device="cuda").bfloat16()
    place = torch.arange(M - 100, M, dtype=torch.int32, device="cuda").view(50, 2)
    share = torch.rand(50, 2, device="cuda")
    check_combine(st.stamp_expert_combine(y, place, share), y[-100:], place - (M - 100), share, None)


def test_arguments_are_checked(st):  # noqa: F811
    import torch
    x = torch.randn(8, 16, device="cuda")
    y, place, share = torch.randn(16, 24, device="cuda"), torch.zeros(8, 2, dtype=torch.int32, device="cuda"), torch.rand(8, 2, device="cuda")
    for bad in (lambda: st.stamp_expert_route(x.half(), 2), lambda: st.stamp_expert_route(x[0], 2), lambda: st.stamp_expert_route(x.t(), 2),
                lambda: st.stamp_expert_route(x, -1), lambda: st.stamp_expert_route(x, 2.0), lambda: st.stamp_expert_route(x, 2, out=(1, 2)),
                lambda: st.stamp_expert_route(x.cpu(), 2), lambda: st.stamp_expert_combine(y.half(), place, share),
                lambda: st.stamp_expert_combine(y, place.long(), share), lambda: st.stamp_expert_combine(y, place, share[:7]),
                lambda: st.stamp_expert_combine(y, place, share, residual=y[:8, :23]), lambda: st.stamp_expert_combine(y.t(), place, share),
                lambda: st.stamp_expert_combine(y, place, share, out_dtype=torch.float16)):
        with pytest.raises(ValueError):
            bad()
    for status, bad in ((1, lambda: st.stamp_expert_route(x, 0)), (1, lambda: st.stamp_expert_route(x, 17)),
                        (2, lambda: st.stamp_expert_route(torch.zeros(2, 1025, device="cuda"), 2)), (2, lambda: st.stamp_expert_route(torch.zeros(2, 64, device="cuda"), 33)),
                        (1, lambda: st.stamp_expert_combine(y, place[:, :0].contiguous(), share[:, :0].contiguous()))):
        with pytest.raises(st.StampError) as e:
            bad()
        assert e.value.status == status
    assert st.stamp_last_device_status() == 0
