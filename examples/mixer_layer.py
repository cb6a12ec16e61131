"""A transformer layer around the mixer, trained and then run with 8-bit weights.

    h = x + block(norm(x));   y = h + W2 gelu(W1 norm(h) + b1) + b2

The block is W_in, the mixer and W_out; the norms are RMS norms, the second one with the residual's addition, and the two
products carry bias, activation and residual in their epilogues.  Training goes through autograd in bf16; in serving the second
norm writes 8-bit values with a scale a token, and the first product reads them with 8-bit weights.

With --norm layer the norms are layer norms; with --gated the feed-forward half is W2 (silu(Wg norm(h) + bg) (Wu norm(h) + bu)) + b2,
both first products in one kernel; with --max-norm a step's gradients are scaled down to a common norm.

    python examples/mixer_layer.py [--tokens 4096] [--channels 128] [--steps 20] [--norm layer] [--gated] [--max-norm 1.0]
"""
from __future__ import annotations

import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2607_25234_gb300 import whtmix  # noqa: E402


class MixerLayer:
    """Parameters and the calls of one layer: N tokens (a power of two) of C channels; in the feed-forward half 4 C, or gated 8 C / 3 (a
    multiple of 8)."""

    def __init__(self, N: int, C: int, seed: int = 0, device: str = "cuda", norm: str = "rms", gated: bool = False):
        if norm not in ("rms", "layer"):
            raise ValueError(f"norm must be 'rms' or 'layer', got {norm!r}")
        g = torch.Generator(device=device)
        g.manual_seed(seed)

        def weight(rows, cols):
            return (torch.randn(rows, cols, generator=g, device=device) / math.sqrt(cols)).to(torch.bfloat16)

        self.norm, self.gated = norm, gated
        self.norm1, self.norm2 = torch.ones(C, device=device), torch.ones(C, device=device)
        self.shift1, self.shift2 = (torch.zeros(C, device=device), torch.zeros(C, device=device)) if norm == "layer" else (None, None)
        self.w_in, self.w_out = weight(C, C), weight(C, C)
        self.gains = torch.ones(N, C, device=device)
        hidden = (8 * C // 3 + 7) // 8 * 8 if gated else 4 * C
        rows = 2 * hidden if gated else hidden  # gated: the gate's rows, then the value's
        self.w1, self.b1 = weight(rows, C), torch.zeros(rows, device=device)
        self.w2, self.b2 = weight(C, hidden), torch.zeros(C, device=device)
        self.w1_8 = None

    def parameters(self):
        shifts = [self.shift1, self.shift2] if self.norm == "layer" else []
        return [self.norm1, self.norm2, self.w_in, self.w_out, self.gains, self.w1, self.b1, self.w2, self.b2] + shifts

    def train_forward(self, x: torch.Tensor) -> torch.Tensor:
        """y with autograd: every step's forward and backward run in the CUDA library."""
        if self.norm == "layer":
            n, _ = whtmix.LayerNormFunction.apply(x, self.norm1, self.shift1)
        else:
            n, _ = whtmix.RMSNormFunction.apply(x, self.norm1)
        m = whtmix.WHTMixBlockFunction.apply(n, self.w_in, self.gains, self.w_out)
        if self.norm == "layer":
            n, h = whtmix.LayerNormFunction.apply(m, self.norm2, self.shift2, x)
        else:
            n, h = whtmix.RMSNormFunction.apply(m, self.norm2, x)
        if self.gated:
            u = whtmix.GatedLinearFunction.apply(n, self.w1, self.b1, "silu")
        else:
            u = whtmix.LinearFunction.apply(n, self.w1, self.b1, None, "gelu")
        return whtmix.LinearFunction.apply(u, self.w2, self.b2, h)

    def quantize(self) -> None:
        """Lays the first product's weights out in 8 bits, once."""
        self.w1_8, self.w1_scale = whtmix.quantize_rows(self.w1)

    def normed(self, x, gain, shift, **kw):
        return whtmix.layer_norm(x, gain, shift, **kw) if self.norm == "layer" else whtmix.rms_norm(x, gain, **kw)

    def forward(self, x: torch.Tensor) -> torch.Tensor:
        """y without gradients; in 8 bits where the weights have been laid out."""
        n = self.normed(x, self.norm1, self.shift1)
        m = whtmix.block_forward(n, self.w_in, self.gains, self.w_out)
        if self.w1_8 is None:
            n, h = self.normed(m, self.norm2, self.shift2, residual=x)
            w, scales = self.w1, {}
        else:
            n, scale, h = self.normed(m, self.norm2, self.shift2, residual=x, out_dtype=torch.float8_e4m3fn)
            w, scales = self.w1_8, {"x_scale": scale, "w_scale": self.w1_scale}
        u = whtmix.gated_linear(n, w, self.b1, "silu", **scales) if self.gated else whtmix.linear(n, w, self.b1, "gelu", **scales)
        return whtmix.linear(u, self.w2, self.b2, residual=h, out=h)


def train(layer: MixerLayer, x: torch.Tensor, target: torch.Tensor, steps: int, rate: float = 0.2, max_norm: float | None = None):
    """Plain gradient steps on the mean squared error, the gradients scaled down to max_norm where it is given; the losses."""
    losses = []
    for p in layer.parameters():
        p.requires_grad_(True)
    for _ in range(steps):
        y = layer.train_forward(x)
        loss = (y.float() - target).square().mean()
        loss.backward()
        with torch.no_grad():
            grads = [p.grad for p in layer.parameters()]
            if max_norm is not None:
                whtmix.clip_by_global_norm(grads, max_norm, out=grads)
            for p, grad in zip(layer.parameters(), grads):
                p -= rate * grad.to(p.dtype)
                p.grad = None
        losses.append(float(loss.detach()))
    for p in layer.parameters():
        p.requires_grad_(False)
    return losses


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--tokens", type=int, default=4096)
    ap.add_argument("--channels", type=int, default=128, choices=(64, 128, 256))
    ap.add_argument("--steps", type=int, default=20)
    ap.add_argument("--norm", default="rms", choices=("rms", "layer"))
    ap.add_argument("--gated", action="store_true")
    ap.add_argument("--max-norm", type=float, default=None)
    a = ap.parse_args()
    layer = MixerLayer(a.tokens, a.channels, norm=a.norm, gated=a.gated)
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    x = torch.randn(1, a.tokens, a.channels, generator=g, device="cuda").to(torch.bfloat16)
    target = torch.randn(1, a.tokens, a.channels, generator=g, device="cuda")
    losses = train(layer, x, target, a.steps, max_norm=a.max_norm)
    print(f"loss {losses[0]:.4f} -> {losses[-1]:.4f} in {a.steps} steps")
    y = layer.forward(x)
    layer.quantize()
    y8 = layer.forward(x)
    whtmix.sync()
    rel = float((y8.float() - y.float()).norm() / y.float().norm())
    print(f"8-bit first product: output within {rel:.4f} of bf16's (2-norm)")


if __name__ == "__main__":
    main()
