"""What is measured of the block-scaled 8-bit floating point operators: their cases, their plain forms and their definitions.

Activations and weights are held as e4m3 codes with one power-of-two scale (e8m0) per block of 128 input features -- per
token for activations, per 128 x 128 block for weights.  Four operators: the per-token quantizer (optionally gathering
rows, as a dispatch to experts does), the quantizer behind a gated activation, the product with one weight matrix, and
the product with the weights of one expert per run of rows.

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
        # one token of a decode step, entering an MLP-up layer
        {"name": "quantize one token", "op": "quantize", "tokens": 1, "rows": 1, "features": 4096, "gather": False, "dtype": "bf16"},
        # four prompts of 4096 tokens, entering a down projection
        {"name": "quantize prompt", "op": "quantize", "tokens": 16384, "rows": 16384, "features": 14336, "gather": False, "dtype": "bf16"},
        # 4096 prompt tokens sent to four experts each: every row is read where it lies and written in expert order
        {"name": "quantize dispatch", "op": "quantize", "tokens": 4096, "rows": 16384, "features": 2048, "gather": True, "dtype": "bf16"},
        # between the two products of an expert layer: a decode step with a few dozen rows
        {"name": "gated decode", "op": "gated", "rows": 33, "features": 2048, "dtype": "bf16"},
        # the same for a prompt
        {"name": "gated prompt", "op": "gated", "rows": 16384, "features": 4096, "dtype": "bf16"},
        # one token through the MLP-up layer: the weights have to be read, nothing else counts
        {"name": "linear one token", "op": "linear", "rows": 1, "features": 4096, "outputs": 11008, "out": "bf16", "bias": False},
        # a batch of decode steps through the down projection: few output channels, a long sum
        {"name": "linear decode batch", "op": "linear", "rows": 17, "features": 14336, "outputs": 4096, "out": "bf16", "bias": False},
        # two images of 4096 patches through an attention projection of 1152 features
        {"name": "linear patches", "op": "linear", "rows": 8192, "features": 1152, "outputs": 1152, "out": "bf16", "bias": True},
        # a prompt of 2048 tokens through the MLP-up layer
        {"name": "linear prompt", "op": "linear", "rows": 2048, "features": 4096, "outputs": 11008, "out": "bf16", "bias": False},
        # four prompts of 4096 tokens through the down projection: the largest product
        {"name": "linear long prompt", "op": "linear", "rows": 16384, "features": 14336, "outputs": 4096, "out": "bf16", "bias": False},
        # a decode batch of 40 tokens, eight experts each, over 64 experts: a few rows for each, none for some
        {"name": "experts decode", "op": "experts", "tokens": 40, "top": 8, "experts": 64, "features": 2048, "outputs": 4096, "out": "bf16", "bias": False},
        # 4096 prompt tokens, four experts each, over 32 experts: hundreds of rows for most, as uneven as routing makes them
        {"name": "experts prompt", "op": "experts", "tokens": 4096, "top": 4, "experts": 32, "features": 4096, "outputs": 4096, "out": "bf16", "bias": False},
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _features(rng, lo, hi):
    """Input features: a multiple of 16; mostly whole blocks of 128, sometimes a short last block."""
    k = _log_uniform(rng, lo, hi)
    return max(lo, k // 128 * 128) if rng.random() < 0.6 else max(lo, k // 16 * 16)


def _outputs(rng, lo, hi):
    """Output channels: mostly multiples of 128, sometimes any number."""
    n = _log_uniform(rng, lo, hi)
    return max(lo, n // 128 * 128) if rng.random() < 0.6 else n


def draw(rng):
    op = rng.choice(["quantize", "gated", "linear", "linear", "experts", "experts"])
    while True:
        if op == "quantize":
            t = _log_uniform(rng, 1, 16384)
            gather = rng.random() < 0.4
            c = {"op": op, "tokens": t, "rows": t * rng.choice([1, 2, 4]) if gather else t, "features": _features(rng, 512, 14336), "gather": gather,
                 "dtype": rng.choice(["bf16", "bf16", "f32"])}
            small = c["rows"] * c["features"] * (2 if c["dtype"] == "f32" else 1) <= 16384 * 14336
        elif op == "gated":
            c = {"op": op, "rows": _log_uniform(rng, 1, 32768), "features": _features(rng, 256, 11008), "dtype": rng.choice(["bf16", "bf16", "f32"])}
            small = c["rows"] * c["features"] * (2 if c["dtype"] == "f32" else 1) <= 16384 * 4096
        elif op == "linear":
            c = {"op": op, "rows": _log_uniform(rng, 1, 16384), "features": _features(rng, 512, 14336), "outputs": _outputs(rng, 256, 11008),
                 "out": rng.choice(["bf16", "bf16", "f32"]), "bias": rng.random() < 0.3}
            small = c["rows"] * c["features"] * c["outputs"] <= 16384 * 14336 * 4096
        else:
            e = rng.choice([8, 16, 32, 64])
            c = {"op": op, "tokens": _log_uniform(rng, 1, 4096), "top": rng.choice([1, 2, 4, 8]), "experts": e, "features": _features(rng, 512, 4096),
                 "outputs": _outputs(rng, 256, 4096), "out": rng.choice(["bf16", "bf16", "f32"]), "bias": rng.random() < 0.2}
            small = e * c["features"] * c["outputs"] <= 32 * 4096 * 4096 and c["tokens"] * c["top"] <= 16384
        if small:
            return c


def work(case):
    def blocks(k):
        return -(-k // BLOCK)

    op = case["op"]
    if op in ("quantize", "gated"):
        size = 4 if case["dtype"] == "f32" else 2
        m, k = case["rows"], case["features"]
        # a gather reads each token once and one 32-bit index per row
        read = case["tokens"] * k * size + (4 * m if case["gather"] else 0) if op == "quantize" else 2 * m * k * size
        return {"bytes": read + m * k + m * blocks(k), "flops": (2 if op == "quantize" else 6) * m * k}
    size = 4 if case["out"] == "f32" else 2
    k, n = case["features"], case["outputs"]
    weights = n * k + blocks(n) * blocks(k)
    bias = 4 * n if case["bias"] else 0
    if op == "linear":
        m, used = case["rows"], 1
    else:
        m = case["tokens"] * case["top"]
        # experts that get rows: all of them once there are several rows for each; a handful of tokens reach fewer
        used = case["experts"] * (1.0 - (1.0 - 1.0 / case["experts"]) ** m)
    return {"bytes": m * k + m * blocks(k) + used * (weights + bias) + m * n * size, "flops": 2.0 * m * n * k}


# ------------------------------------------------------------------------------------------------ inputs
def _dtype(name):
    return torch.float32 if name == "f32" else torch.bfloat16


def _activations(g, m, k, dtype):
    """Tokens of differing size with a percent of outlier features, as the layers' inputs have them."""
    x = torch.randn(m, k, generator=g, device="cuda", dtype=torch.float32)
    x *= torch.where(torch.rand(k, generator=g, device="cuda") < 0.01, 30.0, 1.0)
    x *= torch.exp2(2.0 * torch.rand(m, 1, generator=g, device="cuda") - 1.0)
    return x.to(dtype)


def _route(g, tokens, top, experts):
    """`top` different experts for every token, some experts more liked than others: rows in expert order."""
    liking = torch.randn(experts, generator=g, device="cuda")
    scores = liking + 1.5 * torch.randn(tokens, experts, generator=g, device="cuda")
    chosen = scores.topk(min(top, experts), dim=1).indices.reshape(-1)
    order = torch.sort(chosen, stable=True).indices
    counts = torch.bincount(chosen, minlength=experts)
    offsets = torch.zeros(experts + 1, dtype=torch.int32, device="cuda")
    offsets[1:] = torch.cumsum(counts, 0)
    return torch.div(order, min(top, experts), rounding_mode="floor").to(torch.int32), offsets, int(counts.max())


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
        codes.append(c[: shape[1], : shape[2]].contiguous())
        scales.append(byte.view(torch.float8_e8m0fnu))
    return torch.stack([c.view(torch.uint8) for c in codes]).view(torch.float8_e4m3fn), \
        torch.stack([s.view(torch.uint8) for s in scales]).view(torch.float8_e8m0fnu)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    op = case["op"]
    s = {"op": op}
    if op == "quantize":
        s["x"] = _activations(g, case["tokens"], case["features"], _dtype(case["dtype"]))
        s["rows"] = None
        if case["gather"]:
            s["rows"] = torch.randint(0, case["tokens"], (case["rows"],), generator=g, device="cuda", dtype=torch.int32)
            s["rows"][: min(case["rows"], case["tokens"])] = torch.randperm(case["tokens"], generator=g, device="cuda")[: case["rows"]].to(torch.int32)
        return s
    if op == "gated":
        s["x"] = _activations(g, case["rows"], 2 * case["features"], _dtype(case["dtype"]))
        return s
    k, n = case["features"], case["outputs"]
    s["out"] = _dtype(case["out"])
    if op == "linear":
        x = _activations(g, case["rows"], k, torch.bfloat16)
        w, ws = _weights(g, (1, n, k))
        s["w"], s["w_scale"] = w[0], ws[0]
        s["bias"] = torch.randn(n, generator=g, device="cuda") if case["bias"] else None
    else:
        rows, s["offsets"], s["most"] = _route(g, case["tokens"], case["top"], case["experts"])
        x = _activations(g, case["tokens"], k, torch.bfloat16)[rows.long()]
        s["w"], s["w_scale"] = _weights(g, (case["experts"], n, k))
        s["bias"] = torch.randn(case["experts"], n, generator=g, device="cuda") if case["bias"] else None
    s["x"], s["x_scale"] = _quantize(x.float())
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
    """What activation codes [.., m, k] with scales [.., m, blocks] stand for, in fp32."""
    return codes.float() * scale.float().repeat_interleave(BLOCK, dim=-1)[..., : codes.shape[-1]]


def _weight_values(codes, scale):
    rows = scale.float().repeat_interleave(BLOCK, dim=-2)[..., : codes.shape[-2], :]
    return codes.float() * rows.repeat_interleave(BLOCK, dim=-1)[..., : codes.shape[-1]]


def _plain(s):
    op = s["op"]
    if op == "quantize":
        x = s["x"] if s["rows"] is None else s["x"][s["rows"].long()]
        return _quantize(x.float())
    if op == "gated":
        gate, up = s["x"].float().chunk(2, dim=1)
        return _quantize(gate / (1.0 + torch.exp(-gate)) * up)
    x, w = _values(s["x"], s["x_scale"]), _weight_values(s["w"], s["w_scale"])
    if op == "linear":
        y = x @ w.t()
        return (y if s["bias"] is None else y + s["bias"]).to(s["out"])
    # every expert's rows padded to the same number, one batched product, the rows taken back out
    experts, most, m = w.shape[0], s["most"], x.shape[0]
    at = torch.arange(m, device=x.device)
    expert = torch.searchsorted(s["offsets"], at.to(torch.int32), right=True) - 1
    at = expert * most + at - s["offsets"].long()[expert]
    padded = x.new_zeros(experts * most, x.shape[1])
    padded[at] = x
    y = torch.bmm(padded.view(experts, most, -1), w.transpose(1, 2))
    if s["bias"] is not None:
        y = y + s["bias"][:, None, :]
    return y.reshape(experts * most, -1)[at].to(s["out"])


def run(state):
    if not own:
        return _plain(state)
    from paper_2510_26771_b200 import binding as st

    s = state
    if s["op"] == "quantize":
        return st.stamp_fp8_quantize(s["x"], rows=s["rows"])
    if s["op"] == "gated":
        return st.stamp_fp8_gated_quantize(s["x"])
    if s["op"] == "linear":
        return st.stamp_fp8_linear(s["x"], s["x_scale"], s["w"], s["w_scale"], bias=s["bias"], out_dtype=s["out"])
    return st.stamp_fp8_linear_grouped(s["x"], s["x_scale"], s["offsets"], s["w"], s["w_scale"], bias=s["bias"], out_dtype=s["out"])


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


def exact(case, seed):
    s = prepare(case, seed)
    if s["op"] == "quantize":
        x = s["x"].double()
        return _define_quantizer(x if s["rows"] is None else x.index_select(0, s["rows"].long()))
    if s["op"] == "gated":
        x = s["x"].double()
        f = x.shape[1] // 2
        return _define_quantizer(x[:, :f] * torch.sigmoid(x[:, :f]) * x[:, f:])
    x = _in_64_bits(s["x"], s["x_scale"], True)
    if s["op"] == "linear":
        y = torch.mm(x, _in_64_bits(s["w"], s["w_scale"], False).t())
        return y if s["bias"] is None else y + s["bias"].double()
    y = x.new_zeros(x.shape[0], case["outputs"])
    ends = s["offsets"].tolist()
    for e in range(case["experts"]):
        if ends[e + 1] > ends[e]:
            y[ends[e]:ends[e + 1]] = torch.mm(x[ends[e]:ends[e + 1]], _in_64_bits(s["w"][e], s["w_scale"][e], False).t())
            if s["bias"] is not None:
                y[ends[e]:ends[e + 1]] += s["bias"][e].double()
    return y
