"""The layer operators on a GPU at the ends of their ranges.  References in float64; the bounds are test_layer_gpu.py's, with the same
derivation."""
import math
import os
import subprocess
import sys

import pytest
import torch

from paper_2607_25234_gb300 import whtmix
from test_layer_gpu import BF, F32, U16, U32, close, phi, rand

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module", autouse=True)
def device():
    whtmix.library()
    torch.cuda.set_device(0)
    yield
    whtmix.sync()


# ---- slopes ----

@pytest.mark.parametrize("act", ["relu", "gelu", "silu"])
@pytest.mark.parametrize("T,K", [(3, 64), (3, 320), (9729, 64), (9729, 200)])
def test_slopes_of_far_preactivations(T, K, act):
    """act'(p) over all that bf16 holds, each value beside ordinary and beside far ones (two channels share a reciprocal): the
    float32 slope within 2^-16.  One token's dy is 1, all others' 0, so that db is the slope and dw its bf16."""
    far = [5.0, 7.5, 10.0, 16.0, 20.0, 41.0, 64.0, 88.0, 100.0, 200.0, 300.0, 1e3, 1e4, 1e5, 1e6, 1e7, 1e9, 1e19, 1e20, 1e30, 3e38, math.inf]
    far = far + [-v for v in far]
    pairs = [(v, a) for v in far for a in [0.3, -1.0, 2.0, -7.0, 1e3, -1e6, math.inf, -math.inf, math.nan] + rand(7, 8).tolist()]
    p = torch.tensor(pairs + [(a, v) for v, a in pairs], device="cuda").to(BF).view(-1)
    N = p.numel()
    ref = phi(p.double(), act)[1]
    ref[p == math.inf], ref[p == -math.inf] = 1.0, 0.0
    if act != "relu":
        ref[torch.isnan(p)] = math.nan
    dy, x = torch.zeros(T, N, device="cuda").to(BF), torch.zeros(T, K, device="cuda").to(BF)
    dy[1], x[1] = 1.0, 1.0
    w = torch.zeros(N, K, device="cuda").to(BF)
    rows = p.expand(T, N).contiguous()
    if act == "relu":
        rows[torch.isnan(rows)] = 0.5
        ref[torch.isnan(p)] = 1.0
    _, dw, db = whtmix.linear_backward(x, w, dy, rows, act)
    close(db, ref, 2.0 ** -16)
    close(dw, ref[:, None].expand(N, K), 2.0 ** -16 + U16 * (1 + U16) * (ref.abs() + 2.0 ** -16)[:, None])


# ---- RMS norm ----

def norm_backward_ref(h, w, dy, eps):
    H, W, G = h.double(), w.double(), dy.double()
    D, T = h.shape[-1], h.shape[0]
    rstd = 1.0 / torch.sqrt(H.square().mean(-1, keepdim=True) + eps)
    a, n = G * W, H * rstd
    dx = rstd * a - H * rstd ** 3 * (a * H).mean(-1, keepdim=True)
    spread = rstd * a.abs() + H.abs() * rstd ** 3 * (a * H).abs().mean(-1, keepdim=True)
    unit = U16 if h.dtype == BF else U32
    dx_bound = unit * (1 + U16) * dx.abs() + ((D / 32 + 80) * U32 + 2.0 ** -19) * spread + 1e-37
    dw_bound = ((T / 32 + D / 32 + 200) * U32 + 2.0 ** -19) * (G * n).abs().sum(0) + 1e-37
    return dx, dx_bound, (G * n).sum(0), dw_bound


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T,D", [(1, 1), (1, 8), (1, 256), (3, 64), (5, 128), (33, 512), (70, 65), (9, 250), (153, 77), (1219, 12), (1300, 177), (2, 5001)])
def test_norm_backward_without_eps(T, D, dtype):
    """eps = 0: rows are not 0, so that every gradient is finite, whatever a CTA's idle row groups hold."""
    w, h, dy = 1.0 + 0.1 * rand(3, D), rand(1, T, D).to(dtype), rand(4, T, D).to(dtype)
    wide = torch.zeros(T, 2 * D + 1, dtype=dtype, device="cuda")
    wide[:, 1:D + 1] = h
    for rows in (h, wide[:, 1:D + 1]):  # and rows at any distance from a 16-byte boundary
        dx, dw = whtmix.rms_norm_backward(rows, w, dy, eps=0.0)
        dx_ref, dx_bound, dw_ref, dw_bound = norm_backward_ref(h, w, dy, 0.0)
        close(dx, dx_ref, dx_bound)
        close(dw, dw_ref, dw_bound)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T,D", [(1, 16392), (3, 20001), (130, 16400), (70, 8200)])
def test_norm_backward_of_long_rows_in_place(T, D, dtype):
    """dx over dy and over dh: dx and dw are those of separate matrices."""
    w, h, dy, dh = 1.0 + 0.1 * rand(3, D), rand(1, T, D).to(dtype), rand(4, T, D).to(dtype), rand(5, T, D).to(dtype)
    for extra in (None, dh):
        dx, dw = whtmix.rms_norm_backward(h, w, dy, dh=extra)
        dx_ref, dx_bound, dw_ref, dw_bound = norm_backward_ref(h, w, dy, 1e-6)
        if extra is None:
            close(dx, dx_ref, dx_bound)
        close(dw, dw_ref, dw_bound)
        a = dy.clone()
        got = whtmix.rms_norm_backward(h, w, a, dh=extra, dx=a)
        assert got[0] is a and torch.equal(a, dx) and torch.equal(got[1], dw)
    b = dh.clone()
    got = whtmix.rms_norm_backward(h, w, dy, dh=b, dx=b)
    assert torch.equal(b, dx) and torch.equal(got[1], dw)


WIDTHS = """
import sys
sys.path[:0] = [{root!r}, {tests!r}]
import torch
from paper_2607_25234_gb300 import whtmix
from test_layer_gpu import close, norm_ref, rand, U16, U32
from test_layer_edges_gpu import norm_backward_ref
dtype = getattr(torch, {dtype!r})
for D in {widths}:
    w, x, dy = 1.0 + 0.1 * rand(3, D), rand(1, 5, D).to(dtype), rand(4, 5, D).to(dtype)
    if {backward}:
        dx, dw = whtmix.rms_norm_backward(x, w, dy)
        dx_ref, dx_bound, dw_ref, dw_bound = norm_backward_ref(x, w, dy, 1e-6)
        close(dx, dx_ref, dx_bound)
        close(dw, dw_ref, dw_bound)
    else:
        y, ref = whtmix.rms_norm(x, w), norm_ref(x, None, w)[1]
        close(y, ref, (U16 * (1 + U16) if dtype == torch.bfloat16 else U32) * ref.abs() + ((D / 32 + 60) * U32 + 2.0 ** -21) * ref.abs() + 1e-37)
whtmix.sync()
print("widths ok")
"""


def widths_in_a_fresh_process(dtype, backward, widths):
    """Unaligned rows of these widths one after another, in a process that has run no others."""
    code = WIDTHS.format(root=ROOT, tests=os.path.join(ROOT, "tests"), dtype=dtype, backward=backward, widths=widths)
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=240)
    assert r.returncode == 0 and "widths ok" in r.stdout, r.stderr[-2000:]


@pytest.mark.parametrize("dtype,backward,widths", [
    ("bfloat16", True, [8001, 6501, 8001, 7001, 8001]), ("float32", True, [8001, 6501, 8001, 7001, 8001]),
    ("bfloat16", False, [16001, 12501, 16001, 14001, 16001])])
def test_odd_widths_in_any_order(dtype, backward, widths):
    """A narrower row's launch leaves a wider one's shared memory."""
    widths_in_a_fresh_process(dtype, backward, widths)


@pytest.mark.parametrize("dtype,backward,widths", [("bfloat16", True, [6115, 6121]), ("bfloat16", True, [6127]), ("float32", True, [6121]),
                                                   ("float32", True, [6135]), ("bfloat16", False, [12257, 12281])])
def test_odd_widths_about_the_default_limit(dtype, backward, widths):
    """The gains and sums alone are at most 48 KB, with the kernel's own shared memory they are more."""
    widths_in_a_fresh_process(dtype, backward, widths)


# ---- empty batches, streams, autograd ----

@pytest.mark.parametrize("lead", [(0,), (0, 4), (3, 0)])
def test_an_empty_batch_and_each_gradient_alone(lead):
    x, w = torch.empty(*lead, 32, dtype=BF, device="cuda"), (rand(2, 64, 32) / 5).to(BF)
    dy = torch.empty(*lead, 64, dtype=BF, device="cuda")
    for act, p in (("none", None), ("gelu", dy)):
        for need in ((True, False, False), (False, True, False), (False, False, True), (True, True, True)):
            dx, dw, db = whtmix.linear_backward(x, w, dy, p, act, *need)
            assert (dx.shape == x.shape) if need[0] else dx is None
            assert bool((dw == 0).all()) and dw.shape == w.shape if need[1] else dw is None
            assert bool((db == 0).all()) and db.shape == (64,) if need[2] else db is None
        xr = x.clone().requires_grad_(True)
        whtmix.LinearFunction.apply(xr, w, None, None, act).sum().backward()
        assert xr.grad.shape == x.shape


def stream_of(t):
    """The stream whose memory t lies in."""
    for s in torch.cuda.memory_snapshot():
        if s["address"] <= t.data_ptr() < s["address"] + s["total_size"]:
            return s["stream"]
    raise AssertionError("not in a segment of the allocator")


def test_results_of_a_call_on_a_stream_are_that_streams():
    """Memory that another stream may still be using, or may take back at once, is not what a call on this stream writes."""
    s = torch.cuda.Stream()
    T, N, K = 300, 256, 200
    gain, w, b = torch.ones(K, device="cuda"), (rand(2, N, K) / 14).to(BF), rand(3, N)
    x, r, dy = rand(1, T, K).to(BF), rand(4, T, K).to(BF), rand(5, T, N).to(BF)
    torch.cuda.synchronize()
    y, h = whtmix.rms_norm(x, gain, residual=r, stream=s)
    q = whtmix.rms_norm(x, gain, residual=r, out_dtype=torch.float8_e4m3fn, stream=s)
    z, p = whtmix.linear(y, w, bias=b, activation="gelu", preact=True, stream=s)
    grads = whtmix.linear_backward(y, w, dy, p, "gelu", stream=s) + whtmix.rms_norm_backward(h, gain, y, stream=s)
    given = torch.empty(T, N, dtype=BF, device="cuda")
    assert whtmix.linear(y, w, out=given, stream=s) is given
    for t in (y, h, *q, z, p, *grads):
        assert stream_of(t) == s.cuda_stream
    whtmix.sync(s)
    want = whtmix.linear(whtmix.rms_norm(x, gain, residual=r)[0], w, bias=b, activation="gelu")
    assert torch.equal(z, want) and torch.cuda.current_stream() != s
    cpu = torch.zeros(2, 16, dtype=BF)
    with pytest.raises(ValueError, match="CUDA"):
        whtmix.rms_norm(cpu, torch.ones(16), stream=s)


def test_norm_function_passes_only_the_gradients_that_arrive(monkeypatch):
    T, D = 40, 48
    x, r, w = rand(1, T, D).to(BF), rand(2, T, D).to(BF), 1.0 + 0.1 * rand(3, D)
    gy, gh = rand(4, T, D).to(BF), rand(5, T, D).to(BF)
    seen = []
    plain = whtmix.rms_norm_backward
    monkeypatch.setattr(whtmix, "rms_norm_backward", lambda h, w, dy, dh=None, **kw: (seen.append(dh is not None), plain(h, w, dy, dh=dh, **kw))[1])
    for residual in (None, r):
        for use_y, use_h in ((True, False), (True, True), (False, True)):
            leaves = [x.clone().requires_grad_(True), w.clone().requires_grad_(True)]
            if residual is not None:
                leaves.append(residual.clone().requires_grad_(True))
            y, h = whtmix.RMSNormFunction.apply(*leaves)
            outs, grads = ([y] if use_y else []) + ([h] if use_h else []), ([gy] if use_y else []) + ([gh] if use_h else [])
            seen.clear()
            torch.autograd.backward(outs, grads)
            if use_y:
                dx, dw = plain(h.detach(), w, gy, dh=gh if use_h else None)
                assert seen == [use_h]
            else:
                dx, dw = gh, torch.zeros_like(w)
                assert seen == []
            assert torch.equal(leaves[0].grad, dx) and torch.equal(leaves[1].grad, dw)
            assert residual is None or torch.equal(leaves[2].grad, dx)


def test_second_derivatives_are_refused():
    """A penalty on a gradient raises: it would have been left out of the second one."""
    x, w = rand(1, 4, 16).to(BF).requires_grad_(True), torch.ones(16, device="cuda", requires_grad=True)
    m = (rand(2, 8, 16) / 4).to(BF).requires_grad_(True)
    for y in (whtmix.RMSNormFunction.apply(x, w)[0], whtmix.LinearFunction.apply(x, m, None, None, "gelu")):
        loss = y.float().square().sum()
        (g,) = torch.autograd.grad(loss, x, create_graph=True)
        with pytest.raises(RuntimeError, match="once_differentiable"):
            (loss + g.float().square().sum()).backward()
