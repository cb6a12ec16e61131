"""The layer of examples/mixer_layer.py on a GPU: its forward against float64 with the roundings of its steps, its gradients
against autograd of the same layer in plain torch, the 8-bit form against the bf16 one, and a few training steps."""
import importlib.util
import math
import os

import pytest
import torch

from paper_2607_25234_gb300 import whtmix

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("mixer_layer", os.path.join(ROOT, "examples", "mixer_layer.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def inputs(layer, B, N, C):
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    for name in ("norm1", "norm2", "gains", "b1", "b2"):
        p = getattr(layer, name)
        p += 0.1 * torch.randn(p.shape, generator=g, device="cuda")
    return torch.randn(B, N, C, generator=g, device="cuda").to(torch.bfloat16), torch.randn(B, N, C, generator=g, device="cuda")


def hadamard(n):
    h = torch.ones(1, 1, dtype=torch.float64, device="cuda")
    while h.shape[0] < n:
        h = torch.cat([torch.cat([h, h], 1), torch.cat([h, -h], 1)], 0)
    return h


def plain(layer, x, params):
    """The layer in float64, without any of the library."""
    norm1, norm2, w_in, w_out, gains, w1, b1, w2, b2 = params
    N, C = gains.shape

    def norm(v, g):
        return v * torch.rsqrt(v.square().mean(-1, keepdim=True) + 1e-6) * g

    HN, HC = hadamard(N), hadamard(C)
    z = norm(x, norm1) @ w_in.T
    m = (HN @ (gains * (HN @ z @ HC)) @ HC / (N * C)) @ w_out.T
    h = x + m
    p = norm(h, norm2) @ w1.T + b1
    c = math.sqrt(2 / math.pi)
    return h + (p * torch.sigmoid(2 * c * (p + 0.044715 * p ** 3))) @ w2.T + b2


@pytest.mark.parametrize("B,N,C", [(2, 256, 64), (1, 1024, 128)])
def test_forward_and_gradients(example, B, N, C):
    layer = example.MixerLayer(N, C)
    x, dy = inputs(layer, B, N, C)
    params = layer.parameters()
    exact = [p.double().requires_grad_(True) for p in params]
    xe = x.double().requires_grad_(True)
    ye = plain(layer, xe, exact)
    (ye * dy.double()).sum().backward()
    for p in params:
        p.requires_grad_(True)
    xr = x.clone().requires_grad_(True)
    y = layer.train_forward(xr)
    # about ten bf16 roundings of activations on the way, each 2^-8 of a value at most: the bf16 tolerance 1e-2 in the 2-norm
    assert float((y.detach().double() - ye.detach()).norm() / ye.detach().norm()) <= 1e-2
    (y.float() * dy.to(torch.bfloat16).float()).sum().backward()
    for got, want in zip([xr] + params, [xe] + exact):
        rel = float((got.grad.double() - want.grad).norm() / want.grad.norm())
        assert rel <= 2e-2, rel  # the forward's and the backward's roundings together
    for p in params:
        p.requires_grad_(False)
    out = layer.forward(x)
    assert torch.equal(out, y.detach())
    layer.quantize()
    out8 = layer.forward(x)
    # e4m3 rounds each activation and weight by 2^-5 of it on average at most: the first product's error is that, one half of y
    assert float((out8.double() - ye.detach()).norm() / ye.detach().norm()) <= 6e-2
    whtmix.sync()


def test_training_lowers_the_loss(example):
    layer = example.MixerLayer(512, 64)
    x, target = inputs(layer, 1, 512, 64)
    losses = example.train(layer, x, target, 10)
    assert losses[-1] < losses[0] and all(math.isfinite(v) for v in losses)
