"""A transformer layer around the mixer, trained and then run with 8-bit weights.

    h = x + block(norm(x));   y = h + W2 gelu(W1 norm(h) + b1) + b2

The block is W_in, the mixer and W_out; the norms are RMS norms, the second one with the residual's addition, and the two
products carry bias, activation and residual in their epilogues.  Training goes through autograd in bf16; in serving the second
norm writes 8-bit values with a scale a token, and the first product reads them with 8-bit weights.

    python examples/mixer_layer.py [--tokens 4096] [--channels 128] [--steps 20]
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
    """Parameters and the calls of one layer: N tokens (a power of two) of C channels, 4 C in the feed-forward half."""

    def __init__(self, N: int, C: int, seed: int = 0, device: str = "cuda"):
        g = torch.Generator(device=device)
        g.manual_seed(seed)

        def weight(rows, cols):
            return (torch.randn(rows, cols, generator=g, device=device) / math.sqrt(cols)).to(torch.bfloat16)

        self.norm1, self.norm2 = torch.ones(C, device=device), torch.ones(C, device=device)
        self.w_in, self.w_out = weight(C, C), weight(C, C)
        self.gains = torch.ones(N, C, device=device)
        self.w1, self.b1 = weight(4 * C, C), torch.zeros(4 * C, device=device)
        self.w2, self.b2 = weight(C, 4 * C), torch.zeros(C, device=device)
        self.w1_8 = None

    def parameters(self):
        return [self.norm1, self.norm2, self.w_in, self.w_out, self.gains, self.w1, self.b1, self.w2, self.b2]

    def train_forward(self, x: torch.Tensor) -> torch.Tensor:
        """y with autograd: every step's forward and backward run in the CUDA library."""
        n, _ = whtmix.RMSNormFunction.apply(x, self.norm1)
        m = whtmix.WHTMixBlockFunction.apply(n, self.w_in, self.gains, self.w_out)
        n, h = whtmix.RMSNormFunction.apply(m, self.norm2, x)
        u = whtmix.LinearFunction.apply(n, self.w1, self.b1, None, "gelu")
        return whtmix.LinearFunction.apply(u, self.w2, self.b2, h)

    def quantize(self) -> None:
        """Lays the first product's weights out in 8 bits, once."""
        self.w1_8, self.w1_scale = whtmix.quantize_rows(self.w1)

    def forward(self, x: torch.Tensor) -> torch.Tensor:
        """y without gradients; in 8 bits where the weights have been laid out."""
        n = whtmix.rms_norm(x, self.norm1)
        m = whtmix.block_forward(n, self.w_in, self.gains, self.w_out)
        if self.w1_8 is None:
            n, h = whtmix.rms_norm(m, self.norm2, residual=x)
            u = whtmix.linear(n, self.w1, self.b1, "gelu")
        else:
            q, scale, h = whtmix.rms_norm(m, self.norm2, residual=x, out_dtype=torch.float8_e4m3fn)
            u = whtmix.linear(q, self.w1_8, self.b1, "gelu", x_scale=scale, w_scale=self.w1_scale)
        return whtmix.linear(u, self.w2, self.b2, residual=h, out=h)


def train(layer: MixerLayer, x: torch.Tensor, target: torch.Tensor, steps: int, rate: float = 0.2):
    """Plain gradient steps on the mean squared error; the losses."""
    losses = []
    for p in layer.parameters():
        p.requires_grad_(True)
    for _ in range(steps):
        y = layer.train_forward(x)
        loss = (y.float() - target).square().mean()
        loss.backward()
        with torch.no_grad():
            for p in layer.parameters():
                p -= rate * p.grad.to(p.dtype)
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
    a = ap.parse_args()
    layer = MixerLayer(a.tokens, a.channels)
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    x = torch.randn(1, a.tokens, a.channels, generator=g, device="cuda").to(torch.bfloat16)
    target = torch.randn(1, a.tokens, a.channels, generator=g, device="cuda")
    losses = train(layer, x, target, a.steps)
    print(f"loss {losses[0]:.4f} -> {losses[-1]:.4f} in {a.steps} steps")
    y = layer.forward(x)
    layer.quantize()
    y8 = layer.forward(x)
    whtmix.sync()
    rel = float((y8.float() - y.float()).norm() / y.float().norm())
    print(f"8-bit first product: output within {rel:.4f} of bf16's (2-norm)")


if __name__ == "__main__":
    main()
