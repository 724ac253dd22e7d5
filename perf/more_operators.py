"""What is measured of the operators around the block-scaled products: their cases, their plain forms and their definitions.

  fused      a block-scaled e4m3 product with bias, activation and residual in its epilogue, stored as bf16 or fp32
  quantized  the same product whose activated outputs are quantized again: the next layer's e4m3 codes and scales
  experts    a whole expert layer for a few tokens: for each token, the weighted sum over its experts of
             down(silu(gate(x)) * up(x)), from e4m3 weights and activations as they are, plus a residual
  route      the router's choice: the `top` largest logits of every token, their shares, and the rows in expert order
  combine    the way back: each token's rows weighted, summed and added to a residual

`run` computes an operator from the state that `prepare` made: in its plain form, with elementary torch operations in 32
bits, or, where `own` is true, through the framework's calls.
"""
import math

import torch

own = False

BLOCK = 128
E4M3_MAX = 448.0


# ------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # one token of a decode step through an MLP-up layer with bias and silu: its weights have to be read
        {"name": "fused one token", "op": "fused", "rows": 1, "features": 4096, "outputs": 11008, "act": "silu", "bias": True, "residual": "none", "out": "bf16"},
        # the down projection of two images of 4096 patches, added to the stream that goes round it
        {"name": "fused patches down", "op": "fused", "rows": 8192, "features": 4608, "outputs": 1152, "act": "none", "bias": True, "residual": "bf16", "out": "bf16"},
        # four prompts of 4096 tokens through the down projection, the stream held in fp32: the largest product
        {"name": "fused long prompt", "op": "fused", "rows": 16384, "features": 14336, "outputs": 4096, "act": "none", "bias": False, "residual": "f32", "out": "f32"},
        # the up projection of the same patches: bias, gelu, and the codes that the down projection reads
        {"name": "quantized patches up", "op": "quantized", "rows": 8192, "features": 1152, "outputs": 4608, "act": "gelu_tanh", "bias": True},
        # a prompt of 2048 tokens through an MLP-up layer
        {"name": "quantized prompt", "op": "quantized", "rows": 2048, "features": 4096, "outputs": 11008, "act": "silu", "bias": False},
        # a decode step of one sequence through a small expert layer: latency counts
        {"name": "experts one token", "op": "experts", "tokens": 1, "top": 4, "experts": 16, "features": 1152, "hidden": 2048, "dtype": "bf16", "residual": True, "bias": False},
        # thirteen sequences, large experts: the most weights
        {"name": "experts large", "op": "experts", "tokens": 13, "top": 4, "experts": 32, "features": 4096, "hidden": 4096, "dtype": "bf16", "residual": False, "bias": False},
        # a decode batch of 64, eight experts each: a few rows for each expert, many for some
        {"name": "experts batch", "op": "experts", "tokens": 64, "top": 8, "experts": 64, "features": 2048, "hidden": 2048, "dtype": "bf16", "residual": True, "bias": False},
        # one token of a decode step
        {"name": "route one token", "op": "route", "tokens": 1, "experts": 64, "top": 8, "dtype": "f32", "normalize": True, "masked": False},
        # four prompts of 4096 tokens over many experts
        {"name": "route long prompt", "op": "route", "tokens": 16384, "experts": 256, "top": 8, "dtype": "bf16", "normalize": True, "masked": False},
        # a decode batch of 40 tokens, eight experts each
        {"name": "combine decode", "op": "combine", "tokens": 40, "top": 8, "outputs": 2048, "dtype": "f32", "residual": "bf16", "out": "bf16"},
        # 4096 prompt tokens, four experts each
        {"name": "combine prompt", "op": "combine", "tokens": 4096, "top": 4, "outputs": 4096, "dtype": "bf16", "residual": "bf16", "out": "bf16"},
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _features(rng, lo, hi):
    """Features: a multiple of 16; mostly whole blocks of 128, sometimes a short last block."""
    k = _log_uniform(rng, lo, hi)
    return max(lo, k // 128 * 128) if rng.random() < 0.6 else max(lo, k // 16 * 16)


def _outputs(rng, lo, hi):
    """Output channels: mostly multiples of 128, sometimes any number."""
    n = _log_uniform(rng, lo, hi)
    return max(lo, n // 128 * 128) if rng.random() < 0.6 else n


def draw(rng):
    op = rng.choice(["fused", "fused", "quantized", "experts", "experts", "experts", "route", "combine"])
    while True:
        if op in ("fused", "quantized"):
            c = {"op": op, "rows": _log_uniform(rng, 1, 16384), "features": _features(rng, 512, 14336),
                 "outputs": _outputs(rng, 256, 11008) if op == "fused" else _features(rng, 256, 11008),
                 "act": rng.choice(["none", "relu", "gelu", "gelu_tanh", "silu"]), "bias": rng.random() < 0.5}
            if op == "fused":
                c["residual"], c["out"] = rng.choice(["none", "bf16", "bf16", "f32"]), rng.choice(["bf16", "bf16", "f32"])
            small = c["rows"] * c["features"] * c["outputs"] <= 16384 * 14336 * 4096
        elif op == "experts":
            c = {"op": op, "tokens": _log_uniform(rng, 1, 64), "top": rng.choice([1, 2, 4, 8]), "experts": rng.choice([8, 16, 32, 60, 64, 128]),
                 "features": _features(rng, 512, 4096), "hidden": _features(rng, 256, 4096), "dtype": rng.choice(["bf16", "bf16", "bf16", "f32"]),
                 "residual": rng.random() < 0.5, "bias": rng.random() < 0.2}
            small = c["experts"] * c["features"] * c["hidden"] <= 32 * 4096 * 4096
        elif op == "route":
            c = {"op": op, "tokens": _log_uniform(rng, 1, 16384), "experts": rng.choice([8, 16, 32, 60, 64, 128, 160, 256]), "top": rng.choice([1, 2, 4, 6, 8]),
                 "dtype": rng.choice(["bf16", "f32"]), "normalize": rng.random() < 0.7, "masked": rng.random() < 0.3}
            small = True
        else:
            c = {"op": op, "tokens": _log_uniform(rng, 1, 16384), "top": rng.choice([1, 2, 4, 6, 8]), "outputs": _outputs(rng, 256, 8192),
                 "dtype": rng.choice(["bf16", "f32"]), "residual": rng.choice(["none", "bf16", "f32"]), "out": rng.choice(["bf16", "bf16", "f32"])}
            small = c["tokens"] * c["top"] * c["outputs"] <= 16384 * 8 * 4096
        if small:
            return c


def _size(name):
    return {"none": 0, "bf16": 2, "f32": 4}[name]


def work(case):
    def blocks(k):
        return -(-k // BLOCK)

    op = case["op"]
    if op in ("fused", "quantized"):
        m, k, n = case["rows"], case["features"], case["outputs"]
        read = m * k + m * blocks(k) + n * k + blocks(n) * blocks(k) + (4 * n if case["bias"] else 0)
        if op == "fused":
            return {"bytes": read + m * n * (_size(case["residual"]) + _size(case["out"])), "flops": 2.0 * m * n * k}
        return {"bytes": read + m * n + m * blocks(n), "flops": 2.0 * m * n * k}
    if op == "experts":
        t, e, k, f = case["tokens"], case["experts"], case["features"], case["hidden"]
        m = t * min(case["top"], e)
        # experts that get rows: a handful of tokens do not reach all of them
        used = max(min(case["top"], e), e * (1.0 - (1.0 - 1.0 / e) ** m))
        weights = 3 * k * f + blocks(2 * f) * blocks(k) + blocks(k) * blocks(f) + (4 * (2 * f + k) if case["bias"] else 0)
        tokens = t * k * _size(case["dtype"]) * (3 if case["residual"] else 2)
        return {"bytes": used * weights + tokens + 8 * m + 4 * (e + 1), "flops": 6.0 * m * k * f}
    if op == "route":
        t, e, top = case["tokens"], case["experts"], min(case["top"], case["experts"])
        # logits; then choice, share, row, place and the share by row, and every expert's first row
        return {"bytes": t * e * _size(case["dtype"]) + 20 * t * top + 4 * (e + 1), "flops": 4.0 * t * e}
    t, n = case["tokens"], case["outputs"]
    return {"bytes": t * case["top"] * (n * _size(case["dtype"]) + 8) + t * n * (_size(case["residual"]) + _size(case["out"])), "flops": 2.0 * t * case["top"] * n}


# ------------------------------------------------------------------------------------------------ inputs
def _dtype(name):
    return torch.float32 if name == "f32" else torch.bfloat16


def _activations(g, m, k, dtype):
    """Tokens of differing size with a percent of outlier features, as the layers' inputs have them."""
    x = torch.randn(m, k, generator=g, device="cuda", dtype=torch.float32)
    x *= torch.where(torch.rand(k, generator=g, device="cuda") < 0.01, 30.0, 1.0)
    x *= torch.exp2(2.0 * torch.rand(m, 1, generator=g, device="cuda") - 1.0)
    return x.to(dtype)


def _weights(g, shape):
    """e4m3 codes and e8m0 scales of N(0, 0.02) weights, a scale for each block of 128 x 128."""
    codes, scales = [], []
    for _ in range(shape[0]):
        w = 0.02 * torch.randn(shape[1], shape[2], generator=g, device="cuda")
        n, k = -(-shape[1] // BLOCK), -(-shape[2] // BLOCK)
        p = torch.zeros(n * BLOCK, k * BLOCK, device="cuda")
        p[: shape[1], : shape[2]] = w
        p = p.view(n, BLOCK, k, BLOCK)
        byte, inverse = _scale_of(p.abs().amax(dim=(1, 3)))
        c = (p * inverse[:, None, :, None]).to(torch.float8_e4m3fn).view(n * BLOCK, k * BLOCK)
        codes.append(c[: shape[1], : shape[2]].contiguous().view(torch.uint8))
        scales.append(byte)
    return torch.stack(codes).view(torch.float8_e4m3fn), torch.stack(scales).view(torch.float8_e8m0fnu)


def _logits(g, tokens, experts, dtype, masked):
    """Some experts are more liked than others; masked: a group of them is closed to every token, and some tokens are padding."""
    x = torch.randn(experts, generator=g, device="cuda") + 1.5 * torch.randn(tokens, experts, generator=g, device="cuda")
    if masked:
        x[:, torch.rand(experts, generator=g, device="cuda") < 0.3] = -math.inf
        x[torch.rand(tokens, generator=g, device="cuda") < 0.1] = -math.inf
    return x.to(dtype)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    op = case["op"]
    s = {"op": op}
    if op in ("fused", "quantized"):
        m, k, n = case["rows"], case["features"], case["outputs"]
        s["x"], s["x_scale"] = _quantize(_activations(g, m, k, torch.bfloat16).float())
        w, ws = _weights(g, (1, n, k))
        s["w"], s["w_scale"], s["act"] = w[0], ws[0], case["act"]
        s["bias"] = torch.randn(n, generator=g, device="cuda") if case["bias"] else None
        if op == "fused":
            s["out"] = _dtype(case["out"])
            s["residual"] = None if case["residual"] == "none" else 4.0 * torch.randn(m, n, generator=g, device="cuda").to(_dtype(case["residual"]))
        return s
    if op == "experts":
        t, e, k, f = case["tokens"], case["experts"], case["features"], case["hidden"]
        s["x"] = _activations(g, t, k, _dtype(case["dtype"]))
        _, _, s["rows"], _, s["offsets"], s["row_share"] = _route(_logits(g, t, e, torch.float32, False), min(case["top"], e), True)
        counts = s["offsets"][1:] - s["offsets"][:-1]
        s["used"], s["most"] = torch.nonzero(counts).view(-1), int(counts.max())
        s["up"], s["up_scale"] = _weights(g, (e, 2 * f, k))
        s["down"], s["down_scale"] = _weights(g, (e, k, f))
        s["up_bias"] = torch.randn(e, 2 * f, generator=g, device="cuda") if case["bias"] else None
        s["down_bias"] = torch.randn(e, k, generator=g, device="cuda") if case["bias"] else None
        s["residual"] = _activations(g, t, k, _dtype(case["dtype"])) if case["residual"] else None
        return s
    if op == "route":
        s["logits"] = _logits(g, case["tokens"], case["experts"], _dtype(case["dtype"]), case["masked"])
        s["top"], s["normalize"] = min(case["top"], case["experts"]), case["normalize"]
        return s
    t, top, n = case["tokens"], case["top"], case["outputs"]
    s["y"] = torch.randn(t * top, n, generator=g, device="cuda").to(_dtype(case["dtype"]))
    share = torch.rand(t, top, generator=g, device="cuda")
    s["share"] = share / share.sum(dim=1, keepdim=True)
    s["place"] = torch.randperm(t * top, generator=g, device="cuda").to(torch.int32).view(t, top)
    s["residual"] = None if case["residual"] == "none" else torch.randn(t, n, generator=g, device="cuda").to(_dtype(case["residual"]))
    s["out"] = _dtype(case["out"])
    return s


# ------------------------------------------------------------------------------------------------ plain forms
def _scale_of(amax):
    """The e8m0 byte of the smallest power of two >= 2^-126 that brings amax (fp32) to at most 448, and the scale's
    inverse: from the exponent and mantissa of amax, 448 being 1.75 * 2^8.  1 for a block of zeros, NaN for one that
    is not finite."""
    bits = amax.view(torch.int32)
    e = (bits >> 23) - 135 + ((bits & 0x7FFFFF) > 0x600000).to(torch.int32)
    e = torch.where(bits == 0, 0, e.clamp(min=-126))
    inverse = ((127 - e) << 23).view(torch.float32)
    fine = bits < 0x7F800000
    return torch.where(fine, e + 127, 255).to(torch.uint8), torch.where(fine, inverse, float("nan"))


def _quantize(x):
    """Codes and scales of fp32 rows, a scale for each block of 128 features."""
    m, k = x.shape
    blocks = -(-k // BLOCK)
    if k % BLOCK:
        x = torch.cat([x, x.new_zeros(m, blocks * BLOCK - k)], dim=1)
    x = x.view(m, blocks, BLOCK)
    byte, inverse = _scale_of(x.abs().amax(dim=2))
    codes = (x * inverse[:, :, None]).to(torch.float8_e4m3fn).view(m, blocks * BLOCK)
    return (codes[:, :k].contiguous() if k % BLOCK else codes), byte.view(torch.float8_e8m0fnu)


def _values(codes, scale):
    """What activation codes [m, k] with scales [m, blocks] stand for, in fp32."""
    return codes.float() * scale.float().repeat_interleave(BLOCK, dim=-1)[..., : codes.shape[-1]]


def _weight_values(codes, scale):
    rows = scale.float().repeat_interleave(BLOCK, dim=-2)[..., : codes.shape[-2], :]
    return codes.float() * rows.repeat_interleave(BLOCK, dim=-1)[..., : codes.shape[-1]]


def _activate(z, name):
    if name == "relu":
        return torch.clamp(z, min=0.0)
    if name == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    if name == "gelu_tanh":
        return 0.5 * z * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z * z * z)))
    if name == "silu":
        return z / (1.0 + torch.exp(-z))
    return z


def _route(logits, top, normalize):
    """The `top` largest logits of every token (of equal ones the lower index), their softmax over all experts or over the
    chosen ones; the rows (token, choice) in expert order: each row's token, where each (token, choice) went, every expert's
    first row, each row's share.  A token whose logits are all -inf has shares of zero."""
    tokens, experts = logits.shape
    order = torch.sort(logits, dim=1, descending=True, stable=True)
    chosen, best = order.indices[:, :top], order.values[:, :top].float()
    largest = best[:, :1]
    dead = largest == -math.inf
    weight = torch.exp(best - torch.where(dead, 0.0, largest))
    total = weight.sum(dim=1, keepdim=True) if normalize else torch.exp(logits.float() - torch.where(dead, 0.0, largest)).sum(dim=1, keepdim=True)
    share = weight / torch.where(dead, 1.0, total)
    flat = chosen.reshape(-1)
    order = torch.sort(flat, stable=True).indices
    place = torch.empty_like(order)
    place[order] = torch.arange(order.numel(), device=order.device)
    offsets = torch.zeros(experts + 1, dtype=torch.int32, device=logits.device)
    offsets[1:] = torch.cumsum(torch.bincount(flat, minlength=experts), 0)
    rows = torch.div(order, top, rounding_mode="floor")
    return (chosen.to(torch.int32).contiguous(), share, rows.to(torch.int32), place.to(torch.int32).view(tokens, top), offsets, share.reshape(-1)[order])


def _experts(s):
    """Every used expert's rows padded to the same number, batched products, the rows taken back out and summed by token."""
    used, most, m, t = s["used"], s["most"], s["rows"].numel(), s["x"].shape[0]
    at = torch.arange(m, device=used.device)
    expert = torch.searchsorted(s["offsets"], at.to(torch.int32), right=True) - 1
    slot = torch.searchsorted(used, expert)
    at = slot * most + at - s["offsets"].long()[expert]
    x = s["x"].float()[s["rows"].long()]
    padded = x.new_zeros(used.numel() * most, x.shape[1])
    padded[at] = x

    def pick(v):
        return v.view(torch.uint8)[used].view(v.dtype)

    z = torch.bmm(padded.view(used.numel(), most, -1), _weight_values(pick(s["up"]), pick(s["up_scale"])).transpose(1, 2))
    if s["up_bias"] is not None:
        z = z + s["up_bias"][used][:, None, :]
    gate, up = z.chunk(2, dim=2)
    y = torch.bmm(gate / (1.0 + torch.exp(-gate)) * up, _weight_values(pick(s["down"]), pick(s["down_scale"])).transpose(1, 2))
    if s["down_bias"] is not None:
        y = y + s["down_bias"][used][:, None, :]
    y = y.reshape(used.numel() * most, -1)[at] * s["row_share"][:, None]
    out = s["residual"].float() if s["residual"] is not None else x.new_zeros(t, y.shape[1])
    return out.index_add(0, s["rows"].long(), y).to(s["x"].dtype)


def _plain(s):
    op = s["op"]
    if op in ("fused", "quantized"):
        z = _values(s["x"], s["x_scale"]) @ _weight_values(s["w"], s["w_scale"]).t()
        y = _activate(z if s["bias"] is None else z + s["bias"], s["act"])
        if op == "quantized":
            return _quantize(y)
        return (y if s["residual"] is None else y + s["residual"].float()).to(s["out"])
    if op == "experts":
        return _experts(s)
    if op == "route":
        return _route(s["logits"], s["top"], s["normalize"])
    y = (s["y"].float()[s["place"].long()] * s["share"][:, :, None]).sum(dim=1)
    return (y if s["residual"] is None else y + s["residual"].float()).to(s["out"])


def run(state):
    if not own:
        return _plain(state)
    from paper_2510_26771_b200 import binding as st

    s = state
    if s["op"] in ("fused", "quantized"):
        act = {"none": st.ACT_NONE, "relu": st.ACT_RELU, "gelu": st.ACT_GELU, "gelu_tanh": st.ACT_GELU_TANH, "silu": st.ACT_SILU}[s["act"]]
        if s["op"] == "quantized":
            return st.stamp_fp8_linear_quantized(s["x"], s["x_scale"], s["w"], s["w_scale"], bias=s["bias"], activation=act)
        return st.stamp_fp8_linear_fused(s["x"], s["x_scale"], s["w"], s["w_scale"], bias=s["bias"], activation=act, residual=s["residual"], out_dtype=s["out"])
    if s["op"] == "experts":
        return st.stamp_fp8_expert_layer(s["x"], s["rows"], s["row_share"], s["offsets"], s["up"], s["up_scale"], s["down"], s["down_scale"],
                                         up_bias=s["up_bias"], down_bias=s["down_bias"], residual=s["residual"])
    if s["op"] == "route":
        return st.stamp_expert_route(s["logits"], s["top"], normalize=s["normalize"])
    return st.stamp_expert_combine(s["y"], s["place"], s["share"], residual=s["residual"], out_dtype=s["out"])


# ------------------------------------------------------------------------------------------------ definitions in 64 bits
def _define_quantizer(x):
    """Codes and scales of fp64 rows straight from the definition: scale = the smallest power of two (at least 2^-126)
    with max |x| / scale <= 448, code = x / scale rounded to three mantissa bits (to even), or to multiples of 2^-9
    below 2^-6."""
    m, k = x.shape
    blocks = (k + BLOCK - 1) // BLOCK
    codes, scales = torch.empty_like(x), x.new_empty(m, blocks)
    for b in range(blocks):
        part = x[:, b * BLOCK:(b + 1) * BLOCK]
        mantissa, exponent = torch.frexp(part.abs().max(dim=1).values / E4M3_MAX)
        exponent = torch.where(mantissa == 0.5, exponent - 1, exponent).clamp(min=-126)
        exponent = torch.where(mantissa == 0, torch.zeros_like(exponent), exponent)
        scales[:, b] = torch.ldexp(torch.ones_like(mantissa), exponent)
        v = part / scales[:, b:b + 1]
        step = torch.ldexp(torch.ones_like(v), (torch.frexp(v)[1] - 4).clamp(min=-9))
        codes[:, b * BLOCK:(b + 1) * BLOCK] = torch.round(v / step) * step
    return codes, scales


def _in_64_bits(codes, scale, by_row):
    v = codes.double()
    for b in range(scale.shape[-1]):
        f = scale[..., b].double()
        v[:, b * BLOCK:(b + 1) * BLOCK] *= f[:, None] if by_row else torch.repeat_interleave(f, BLOCK)[: v.shape[0], None]
    return v


def _define_activation(z, name):
    # (by other identities than the plain form's: the complementary error function, and tanh as a logistic function)
    if name == "gelu":
        return z * 0.5 * torch.erfc(-z / math.sqrt(2.0))
    if name == "gelu_tanh":
        return z * torch.sigmoid(2.0 * math.sqrt(2.0 / math.pi) * (z + 0.044715 * z ** 3))
    if name == "silu":
        return z * torch.sigmoid(z)
    return torch.maximum(z, torch.zeros_like(z)) if name == "relu" else z


def _define_route(logits, top, normalize):
    """Token by token: the best expert is looked for `top` times among those that are left."""
    x = logits.double()
    tokens, experts = x.shape
    left, open_ = x.clone(), torch.ones_like(x, dtype=torch.bool)
    index = torch.arange(experts, device=x.device)
    chosen = torch.empty(tokens, top, dtype=torch.int64, device=x.device)
    for j in range(top):
        best = torch.where(open_, left, -math.inf).max(dim=1, keepdim=True).values
        first = torch.where(open_ & (left == best), index, experts).min(dim=1).values
        chosen[:, j] = first
        open_[torch.arange(tokens, device=x.device), first] = False
    picked = torch.gather(x, 1, chosen)
    share = torch.softmax(picked, dim=1) if normalize else torch.gather(torch.softmax(x, dim=1), 1, chosen)
    share = torch.where((x == -math.inf).all(dim=1, keepdim=True), 0.0, share)
    key = chosen.reshape(-1) * (tokens * top) + torch.arange(tokens * top, device=x.device)
    order = torch.argsort(key)
    counts = (chosen.reshape(-1, 1) == index).sum(dim=0) if tokens * top * experts < (1 << 28) else torch.bincount(chosen.reshape(-1), minlength=experts)
    offsets = torch.cat([counts.new_zeros(1), counts.cumsum(0)])
    return (chosen.to(torch.int32), share, (order // top).to(torch.int32), torch.argsort(order).to(torch.int32).view(tokens, top), offsets.to(torch.int32),
            share.reshape(-1)[order])


def exact(case, seed):
    s = prepare(case, seed)
    op = s["op"]
    if op in ("fused", "quantized"):
        z = torch.mm(_in_64_bits(s["x"], s["x_scale"], True), _in_64_bits(s["w"], s["w_scale"], False).t())
        if s["bias"] is not None:
            z += s["bias"].double()
        y = _define_activation(z, s["act"])
        if op == "quantized":
            return _define_quantizer(y)
        return y if s["residual"] is None else y + s["residual"].double()
    if op == "experts":
        ends, x = s["offsets"].tolist(), s["x"].double()
        y = torch.zeros_like(x) if s["residual"] is None else s["residual"].double()
        for e in range(case["experts"]):
            if ends[e + 1] == ends[e]:
                continue
            rows = s["rows"][ends[e]:ends[e + 1]].long()
            z = torch.mm(x[rows], _in_64_bits(s["up"][e], s["up_scale"][e], False).t())
            if s["up_bias"] is not None:
                z += s["up_bias"][e].double()
            f = case["hidden"]
            h = torch.mm(z[:, :f] * torch.sigmoid(z[:, :f]) * z[:, f:], _in_64_bits(s["down"][e], s["down_scale"][e], False).t())
            if s["down_bias"] is not None:
                h += s["down_bias"][e].double()
            y[rows] += h * s["row_share"][ends[e]:ends[e + 1], None].double()
        return y
    if op == "route":
        return _define_route(s["logits"], s["top"], s["normalize"])
    y = s["residual"].double() if s["residual"] is not None else s["y"].new_zeros(case["tokens"], case["outputs"], dtype=torch.float64)
    for j in range(case["top"]):
        y = y + s["y"].double()[s["place"][:, j].long()] * s["share"][:, j:j + 1].double()
    return y
