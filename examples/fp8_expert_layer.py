"""An expert layer served with the block-scaled 8-bit floating point calls: a prompt, then single-token decode steps.

    python examples/fp8_expert_layer.py [--tokens 2048] [--features 1152] [--hidden 2048] [--experts 16] [--top 4] [--steps 8]

Each token goes to `top` of the experts; an expert is a gated layer, down(silu(gate(x)) * up(x)).  A prompt: the router's
logits (torch), the choice and the rows in expert order, then four kernels -- the tokens are quantized in expert order (the
dispatch), multiplied with their expert's gate and up weights, activated and quantized again, multiplied with its down
weights -- and each token's rows are weighted and summed.  A decode step of up to 64 tokens: logits, choice, and one call for
all that follows, on activations that stay as they are.  Weights are random.  The printed errors compare with the layer on
the unquantized weights in fp32.
"""
import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch  # noqa: E402

from paper_2510_26771_b200 import binding as st  # noqa: E402


class ExpertLayer:
    def __init__(self, features: int, hidden: int, experts: int, top: int, seed: int = 0, device="cuda"):
        g = torch.Generator(device=device).manual_seed(seed)
        self.top, self.experts = top, experts
        self.router = torch.randn(features, experts, generator=g, device=device) * features ** -0.5
        # an expert's gates, then its ups: one product for both
        self.up = (torch.randn(experts, 2 * hidden, features, generator=g, device=device) * features ** -0.5).bfloat16()
        self.down = (torch.randn(experts, features, hidden, generator=g, device=device) * hidden ** -0.5).bfloat16()
        self.up_codes, self.up_scale = st.stamp_fp8_quantize_weights(self.up)
        self.down_codes, self.down_scale = st.stamp_fp8_quantize_weights(self.down)

    def route(self, x: torch.Tensor):
        """For every row in expert order its token, where each (token, choice) went, every expert's first row, the weights."""
        _, share, rows, place, offsets, _ = st.stamp_expert_route(x.float() @ self.router, self.top)
        return rows, place, offsets, share

    def __call__(self, x: torch.Tensor) -> torch.Tensor:
        rows, place, offsets, share = self.route(x)
        codes, scale = st.stamp_fp8_quantize(x, rows=rows)
        h = st.stamp_fp8_linear_grouped(codes, scale, offsets, self.up_codes, self.up_scale)
        codes, scale = st.stamp_fp8_gated_quantize(h)
        y = st.stamp_fp8_linear_grouped(codes, scale, offsets, self.down_codes, self.down_scale, out_dtype=torch.float32)
        return st.stamp_expert_combine(y, place, share, out_dtype=x.dtype)

    def decode(self, x: torch.Tensor, residual=None) -> torch.Tensor:
        """Up to 64 tokens, plus what goes round the layer."""
        _, _, rows, _, offsets, row_share = st.stamp_expert_route(x.float() @ self.router, self.top)
        return st.stamp_fp8_expert_layer(x, rows, row_share, offsets, self.up_codes, self.up_scale, self.down_codes, self.down_scale, residual=residual)

    def unquantized(self, x: torch.Tensor) -> torch.Tensor:
        rows, place, offsets, share = self.route(x)
        ends, y = offsets.tolist(), torch.empty(rows.numel(), x.shape[1], device=x.device)
        for e in range(self.experts):
            gate, up = (x[rows[ends[e]:ends[e + 1]].long()].float() @ self.up[e].float().t()).chunk(2, dim=1)
            y[ends[e]:ends[e + 1]] = (torch.nn.functional.silu(gate) * up) @ self.down[e].float().t()
        return (y[place].view(x.shape[0], self.top, -1) * share[:, :, None]).sum(dim=1)


def relative_error(got: torch.Tensor, want: torch.Tensor) -> float:
    return float((got.float() - want).norm() / want.norm())


def main(argv=None) -> dict:
    a = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("tokens", 2048), ("features", 1152), ("hidden", 2048), ("experts", 16), ("top", 4), ("steps", 8)):
        a.add_argument("--" + name, type=int, default=value)
    a = a.parse_args(argv)
    layer = ExpertLayer(a.features, a.hidden, a.experts, a.top)
    g = torch.Generator(device="cuda").manual_seed(1)
    prompt = torch.randn(a.tokens, a.features, generator=g, device="cuda").bfloat16()
    result = {"prompt_error": relative_error(layer(prompt), layer.unquantized(prompt)), "step_errors": []}
    for _ in range(a.steps):
        token = torch.randn(1, a.features, generator=g, device="cuda").bfloat16()
        result["step_errors"].append(relative_error(layer.decode(token), layer.unquantized(token)))
    if st.stamp_last_device_status() != 0:
        raise RuntimeError("device status word raised")
    print(f"prompt of {a.tokens} tokens: relative error {result['prompt_error']:.4f}; "
          f"{a.steps} single tokens: {max(result['step_errors'], default=0.0):.4f} at most")
    return result


if __name__ == "__main__":
    main()
