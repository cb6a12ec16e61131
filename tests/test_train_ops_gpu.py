"""Layer norm, the gated feed-forward half and clipping by a common norm on a GPU, against plain float64 implementations.

Tolerances, derived before any run.  U16 = 2^-8 is the most that rounding to bf16 (8 significand bits) moves a value by, relative to
it; U32 = 2^-24 is float32's.
  * layer norm: a sum of D float32 terms is off by at most S = (D / 32 + 60) U32 of the sum of their magnitudes (a thread adds at most
    D / 32 or 32 terms, then 16 partial sums and shuffles).  h is rounded once (U32 |h|), so that c = h - m is off by
    C = U32 (|h| + |c|) + S mean|h|; the variance by S of itself and by the mean of 2 |c| C + C^2; rstd by half of that, relative, and
    2^-22 (rsqrt).  y takes three more roundings.
  * its gradients: the same C and rstd in n = c rstd, the sums at S, and over T rows at (T / 32 + D / 32 + 200) U32.
  * products: a sum of K terms in float32, the tensor cores' additions truncated: K 2^-23 (|x| |w|^T) element by element.
  * activations: ex2 and rcp at 2^-22, their argument's rounding times the slope of the exponential: 2^-17 |act| + 2^-17 |z slope|;
    slopes 2^-16 where they are used as factors (they are at most 1.13).  The gating multiplies errors: |u| err(act) + |act| err(u).
  * dp is rounded to bf16 before its products: U16 |dp| in each term.
  * the common norm: sums of 64 squares in float32 (66 U32 of a sum of positive terms, half of it in the root), one rounding of the
    norm, one of the factor, one of the product, one to the type.
"""
import importlib.util
import math
import os

import pytest
import torch

from paper_2607_25234_gb300 import whtmix

pytestmark = pytest.mark.gpu

U16, U32 = 2.0 ** -8, 2.0 ** -24
BF, F32, E4M3 = torch.bfloat16, torch.float32, torch.float8_e4m3fn
EPS = 1e-5
ACTS = ["none", "relu", "gelu", "silu"]


@pytest.fixture(scope="module", autouse=True)
def device():
    whtmix.library()
    torch.cuda.set_device(0)
    yield
    whtmix.sync()


def rand(seed, *shape):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randn(*shape, generator=g, device="cuda")


def close(got, ref, bound):
    """|got - ref| <= bound, element by element; NaN and infinities in the same places."""
    got, ref = got.double(), ref.double()
    assert got.shape == ref.shape
    assert torch.equal(torch.isnan(got), torch.isnan(ref))
    fine = torch.isfinite(ref)
    assert torch.equal(torch.isfinite(got), fine)
    worst = ((got - ref).abs() - bound)[fine]
    assert worst.numel() == 0 or float(worst.max()) <= 0, f"beyond its bound by {float(worst.max()):.3e}"


def rounded(ref, err, dtype):
    """The bound of a value that is off by err and then rounded to dtype."""
    unit = U16 if dtype == BF else U32
    return unit * (1 + U16) * (ref.abs() + err) + err + 1e-37


def guarded(shape, dtype):
    """A view into a buffer with guard bytes around it, and a check that they are untouched."""
    n = math.prod(shape) * torch.empty((), dtype=dtype).element_size()
    buf = torch.full((n + 512,), 0x5A, dtype=torch.uint8, device="cuda")
    view = buf[256:256 + n].view(dtype).view(shape)

    def check():
        assert bool((buf[:256] == 0x5A).all()) and bool((buf[256 + n:] == 0x5A).all()), "written outside the output"
    return view, check


# ---- layer norm ----

class Norm:
    """Layer norm in float64 and the bounds of its float32 steps."""

    def __init__(self, h, eps=EPS):
        D = h.shape[-1]
        self.h = h.double()
        mean = lambda v: v.mean(-1, keepdim=True)
        self.sum_err = (D / 32 + 60) * U32
        self.c = self.h - mean(self.h)
        var = mean(self.c.square())
        self.rstd = 1.0 / torch.sqrt(var + eps)
        self.c_err = U32 * (self.h.abs() + self.c.abs()) + self.sum_err * mean(self.h.abs())
        var_err = self.sum_err * var + mean(2 * self.c.abs() * self.c_err + self.c_err.square())
        self.rel = 0.5 * var_err / (var + eps) + 2.0 ** -22
        self.n = self.c * self.rstd
        self.n_err = self.rstd * self.c_err + self.n.abs() * self.rel

    def y(self, w, b):
        w, b = w.double(), 0.0 if b is None else b.double()
        y = self.n * w + b
        return y, w.abs() * self.n_err + 4 * U32 * (self.n * w).abs() + U32 * y.abs()


def norm_inputs(T, D, dtype, offset=0.5):
    x = (rand(1, T, D) + offset * rand(11, D)).to(dtype)
    return x, rand(2, T, D).to(dtype), 1.0 + 0.1 * rand(3, D), 0.1 * rand(4, D)


NORM_SHAPES = [(1, 1), (1, 2), (1, 8), (1, 256), (3, 7), (5, 64), (17, 65), (100, 128), (70, 100), (257, 512), (33, 1000), (64, 1024), (40, 2048),
               (12, 5001), (200, 5000), (7, 8192), (5, 16384), (400, 16), (300, 2999), (5, 8191), (3, 16383), (3, 4097), (700, 77)]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T,D", NORM_SHAPES)
def test_layer_norm_against_float64(T, D, dtype):
    x, res, w, b = norm_inputs(T, D, dtype)
    for residual, shift in ((None, b), (res, b), (res, None)):
        out, out_ok = guarded((T, D), dtype)
        h_out, h_ok = guarded((T, D), dtype) if residual is not None else (None, lambda: None)
        before = x.clone()
        got = whtmix.layer_norm(x, w, shift, residual=residual, out=out, h=h_out)
        ref = Norm(x if residual is None else x.double() + res.double())
        y, err = ref.y(w, shift)
        close(out, y, rounded(y, err, dtype))
        out_ok()
        if residual is not None:
            assert got[0] is out and got[1] is h_out
            close(h_out, ref.h, rounded(ref.h, U32 * ref.h.abs(), dtype))
            h_ok()
        assert torch.equal(x, before)
        plain = whtmix.layer_norm(x, w, shift, residual=residual)  # the compiled way
        assert torch.equal(plain if residual is None else plain[0], out)


def e4m3_step(v):
    """The distance of e4m3 values around v: 2^(e - 3) for |v| in [2^e, 2^(e + 1)), e >= -6, exactly (the exponent's bits)."""
    bits = v.abs().clamp_min(2.0 ** -6).view(torch.int64)
    return ((bits >> 52) - 3 << 52).view(torch.float64)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T,D", NORM_SHAPES + [(2, 20001)])
def test_layer_norm_to_eight_bits(T, D, dtype):
    x, res, w, b = norm_inputs(T, D, dtype)
    q, scale, h = whtmix.layer_norm(x, w, b, residual=res, out_dtype=E4M3)
    assert q.dtype == E4M3 and q.shape == x.shape and scale.shape == (T,)
    y, err = Norm(x.double() + res.double()).y(w, b)
    s = y.abs().amax(-1, keepdim=True) / 448.0
    s_err = err.amax(-1, keepdim=True) / 448.0 + 2 * U32 * s
    close(scale[:, None], s, s_err)
    v = y / s
    v_err = err / s + v.abs() * s_err / s + 4 * U32 * v.abs()
    close(q.float(), v, (e4m3_step(v) / 2 + v_err) * (1 + 2.0 ** -12))
    # all but few are the nearest: those within their error of the middle between two values may go either way
    nearest = (torch.round(v / e4m3_step(v)) * e4m3_step(v)).clamp(-448.0, 448.0)
    assert float((q.double() != nearest).double().mean()) <= 1e-4 + 2.0 / v.numel() + float((v_err / e4m3_step(v)).mean())


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T,D", [(20011, 77), (9800, 33), (10000, 9), (9737, 50), (9729, 67), (4900, 177), (9801, 130), (5000, 301), (2440, 499), (2500, 1001), (2433, 1027), (2500, 1537), (2440, 2047)])
def test_many_odd_rows_to_eight_bits(T, D, dtype):
    """Rows that come as tiles; what lies between the output's rows stays."""
    test_layer_norm_to_eight_bits(T, D, dtype)
    x, res, w, b = norm_inputs(T, D, dtype)
    q, scale, h = whtmix.layer_norm(x, w, b, residual=res, out_dtype=E4M3)
    for gap in (0, 3, 16):
        whole = torch.full((T, D + gap), 0x5a, dtype=torch.uint8, device="cuda")
        out = whole.view(E4M3)[:, :D]
        q2, scale2, h2 = whtmix.layer_norm(x, w, b, residual=res, out_dtype=E4M3, out=out)
        assert torch.equal(q2.view(torch.uint8), q.view(torch.uint8)) and torch.equal(scale2, scale) and torch.equal(h2, h)
        assert bool((whole[:, D:] == 0x5a).all())
    alone, s = whtmix.layer_norm(x, w, out_dtype=E4M3)  # neither residual nor shifts, as each row on its own
    few, s_few = whtmix.layer_norm(x[5:9], w, out_dtype=E4M3)
    assert float((alone[5:9].float() - few.float()).abs().max()) <= 32 and float((s[5:9] - s_few).abs().max()) <= 1e-5 * float(s_few.max())
    x[7, D // 2] = math.inf
    x[8] = 2.5
    odd, s_odd = whtmix.layer_norm(x, w, out_dtype=E4M3)
    assert bool(torch.isnan(s_odd[7])) and bool(torch.isnan(odd[7].float()).all())
    rows = [i for i in range(T) if i not in (7, 8)]
    assert torch.equal(odd.view(torch.uint8)[rows], alone.view(torch.uint8)[rows]) and torch.equal(s_odd[rows], s[rows])
    assert bool((odd[8].float() == 0).all() or float(s_odd[8]) <= 1e-3)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T,D", [(2, 20001), (1, 100000), (3, 33000), (3, 1 << 20)])
def test_layer_norm_of_rows_beyond_the_registers(T, D, dtype):
    x, res, w, b = norm_inputs(T, D, dtype)
    y, h = whtmix.layer_norm(x, w, b, residual=res)
    ref, err = Norm(x.double() + res.double()).y(w, b)
    close(y, ref, rounded(ref, err, dtype))
    check_norm_backward(h, w, rand(5, T, D).to(dtype), None)
    dy = rand(5, T, D).to(dtype)
    want = check_norm_backward(h, w, dy, h)
    over = whtmix.layer_norm_backward(h, w, dy, dh=h.clone(), dx=dy)  # dx in dy's place
    assert all(torch.equal(p, q) for p, q in zip(over, want))


@pytest.mark.parametrize("dtype", [BF, F32])
def test_a_mean_far_from_zero_costs_what_its_rounding_costs(dtype):
    """Channels around 1000 with a deviation of 1: a difference of two sums of squares would leave nothing of the variance."""
    T, D = 50, 1024
    x = (1000.0 + rand(1, T, D)).to(dtype)
    w, b = torch.ones(D, device="cuda"), torch.zeros(D, device="cuda")
    y, err = Norm(x).y(w, b)
    close(whtmix.layer_norm(x, w, b), y, rounded(y, err, dtype))
    check_norm_backward(x, w, rand(5, T, D).to(dtype), None)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_layer_norm_in_place_and_strided(dtype):
    T, D = 65, 1000
    _, r, w, b = norm_inputs(T, D, dtype)
    wide = rand(1, T, 3 * D + 1).to(dtype)
    for start in (0, 1, D + 1):  # aligned and not: the rows' distance is 3 D + 1 elements
        x = wide[:, start:start + D]
        y, h = whtmix.layer_norm(x, w, b, residual=r)
        assert torch.equal(h, whtmix.layer_norm(x.contiguous(), w, b, residual=r)[1])
        ref, err = Norm(x.double() + r.double()).y(w, b)
        close(y, ref, rounded(ref, err, dtype))
    x = rand(1, T, D).to(dtype)
    want_y, want_h = whtmix.layer_norm(x, w, b, residual=r)
    for target in ("x", "r"):
        a, c = x.clone(), r.clone()
        t = a if target == "x" else c
        y, h = whtmix.layer_norm(a, w, b, residual=c, h=t)
        assert h is t and torch.equal(h, want_h) and torch.equal(y, want_y)
        a, c = x.clone(), r.clone()
        t = a if target == "x" else c
        y, h = whtmix.layer_norm(a, w, b, residual=c, out=t)
        assert y is t and torch.equal(h, want_h) and torch.equal(y, want_y)
    # every second row of a wider matrix; what lies between is left alone
    every, mid = torch.full((2 * T, D + 3), 7.0, device="cuda").to(dtype), torch.full((2 * T, D + 3), 7.0, device="cuda").to(E4M3)
    whtmix.layer_norm(x, w, b, out=every[::2, 2:D + 2])
    ref, err = Norm(x).y(w, b)
    close(every[::2, 2:D + 2], ref, rounded(ref, err, dtype))
    every[::2, 2:D + 2] = 7
    assert bool((every == 7).all())
    whtmix.layer_norm(x, w, b, out=mid[1::2, 1:D + 1], out_dtype=E4M3)
    assert bool((mid[::2].float() == 7).all()) and bool((mid[1::2, 0].float() == 7).all()) and bool((mid[1::2, D + 1:].float() == 7).all())
    views = rand(9, 6, 5, 4, 64).to(dtype)[::2, 1]  # [3, 4, 64], two strides
    with pytest.raises(ValueError, match="one stride"):
        whtmix.layer_norm(views, 1.0 + 0.1 * rand(3, 64))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("D", [128, 1001, 20001])
def test_rows_that_are_constant_or_not_finite(D, dtype):
    w, b, T = 1.0 + 0.1 * rand(3, D), 0.1 * rand(4, D), 400 if D < 2000 else 8
    x, dy = rand(1, T, D).to(dtype), rand(5, T, D).to(dtype)
    y0, (dx0, _, _) = whtmix.layer_norm(x, w, b), whtmix.layer_norm_backward(x, w, dy)
    x[0] = 0
    x[1] = 3.0
    x[2, D // 2] = math.inf
    x[3, D - 1] = math.nan
    x[4] *= 1e-20
    y, (dx, dw, db) = whtmix.layer_norm(x, w, b), whtmix.layer_norm_backward(x, w, dy)
    for i in (0, 1):
        close(y[i], b, rounded(b.double(), w.double().abs() * 1e-5 ** -0.5 * 8 * U32 * float(x[i, 0].abs()) * (D / 32 + 60), dtype))
    assert bool(torch.isnan(y[2]).all()) and bool(torch.isnan(y[3]).all())
    ref, err = Norm(x[4:5]).y(w, b)
    close(y[4:5], ref, rounded(ref, err, dtype))
    assert torch.equal(y[5:], y0[5:]) and torch.equal(dx[5:], dx0[5:])  # the neighbours
    assert bool(torch.isnan(dx[2]).all()) and bool(torch.isnan(dx[3]).all()) and bool(torch.isnan(dw).all()) and bool(torch.isfinite(db).all())
    q, scale = whtmix.layer_norm(x, w, None, out_dtype=E4M3)
    assert float(scale[0]) == 0.0 and bool((q[0].float() == 0).all()) and torch.isnan(scale[2]) and torch.isnan(scale[3])
    assert bool(torch.isfinite(scale[4:]).all())
    # one channel: the sum is the mean
    one = whtmix.layer_norm(rand(1, 9, 1).to(dtype), torch.ones(1, device="cuda"), torch.full((1,), 2.0, device="cuda"))
    assert bool((one == 2).all())


def check_norm_backward(h, w, dy, dh):
    T, D = h.shape
    outs = [guarded((T, D), h.dtype), guarded((D,), F32), guarded((D,), F32)]
    dx, dw, db = whtmix.layer_norm_backward(h, w, dy, dh=dh, dx=outs[0][0], dw=outs[1][0], db=outs[2][0])
    for _, ok in outs:
        ok()
    ref = Norm(h)
    mean = lambda v: v.mean(-1, keepdim=True)
    G = dy.double()
    a = G * w.double()
    n, n_err, an = ref.n, ref.n_err, a * ref.n
    want = ref.rstd * (a - mean(a) - n * mean(an))
    spread = ref.rstd * (a.abs() + mean(a.abs()) + n.abs() * mean(an.abs()))
    # n in the products, rstd in all of it, the sums, a few roundings
    err = ref.rstd * (n_err * mean(an.abs()) + n.abs() * mean(a.abs() * n_err)) + (3 * ref.rel + ref.sum_err + 12 * U32) * spread
    if dh is not None:
        want = want + dh.double()
        err = err + U32 * (dh.double().abs() + spread)
    close(dx, want, rounded(want, err, h.dtype))
    rows = (T / 32 + D / 32 + 200) * U32
    close(dw, (G * n).sum(0), rows * (G * n).abs().sum(0) + (G.abs() * n_err).sum(0) + 4 * U32 * (G * n).abs().sum(0) + 1e-37)
    close(db, G.sum(0), rows * G.abs().sum(0) + 1e-37)
    return dx, dw, db


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T,D", NORM_SHAPES + [(3001, 64), (1500, 257), (20011, 77), (2433, 1001), (5000, 9), (1217, 177), (20003, 33), (9, 12000)])
def test_layer_norm_backward_against_float64(T, D, dtype):
    h, _, w, _ = norm_inputs(T, D, dtype)
    dy, dh = rand(5, T, D).to(dtype), rand(6, T, D).to(dtype)
    check_norm_backward(h, w, dy, None)
    dx, dw, db = check_norm_backward(h, w, dy, dh)
    again = whtmix.layer_norm_backward(h, w, dy, dh=dh)
    assert all(torch.equal(p, q) for p, q in zip(again, (dx, dw, db)))  # a fixed order of additions
    part = whtmix.layer_norm_backward(h, w, dy, dh=dh, need_db=False)
    assert torch.equal(part[0], dx) and torch.equal(part[1], dw) and part[2] is None
    for inplace in ("dy", "dh"):
        a, b = dy.clone(), dh.clone()
        got = whtmix.layer_norm_backward(h, w, a, dh=b, dx=a if inplace == "dy" else b)
        assert all(torch.equal(p, q) for p, q in zip(got, (dx, dw, db)))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T,D", [(2433, 1027), (2500, 1373), (2441, 1537), (2440, 2047)])
def test_layer_norm_of_many_wide_odd_rows(T, D, dtype):
    test_layer_norm_against_float64(T, D, dtype)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T,D", [(2433, 529), (2500, 601), (2441, 765), (4999, 1021), (2440, 1277), (2600, 1502), (2433, 2047), (2435, 1135)])
def test_layer_norm_backward_of_many_wide_odd_rows(T, D, dtype):
    test_layer_norm_backward_against_float64(T, D, dtype)
    h, w, dy, dh = rand(1, T, D).to(dtype), 1 + 0.1 * rand(2, D), rand(3, T, D).to(dtype), rand(4, T, D).to(dtype)
    for extra in (None, dh):
        want = whtmix.layer_norm_backward(h, w, dy, dh=extra)
        over = dy.clone()
        got = whtmix.layer_norm_backward(h, w, over, dh=extra, dx=over)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        if extra is not None:
            over = dh.clone()
            got = whtmix.layer_norm_backward(h, w, dy, dh=over, dx=over)
            assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_layer_norm_gradients_by_differences():
    T, D = 3, 24
    x, r, w, b = rand(1, T, D) + 1.0, rand(2, T, D), 1.0 + 0.1 * rand(3, D), 0.1 * rand(4, D)
    dy, dh = rand(5, T, D), rand(6, T, D)

    def loss(x_, w_, b_):
        h = x_ + r.double()
        return float(((h - h.mean(-1, keepdim=True)) / torch.sqrt(h.var(-1, keepdim=True, unbiased=False) + EPS) * w_ + b_).mul(dy.double()).sum()
                     + (h * dh.double()).sum())

    leaves = [t.clone().requires_grad_(True) for t in (x, w, b, r)]
    y, h = whtmix.LayerNormFunction.apply(leaves[0], leaves[1], leaves[2], leaves[3], EPS)
    ((y * dy).sum() + (h * dh).sum()).backward()
    assert torch.equal(leaves[0].grad, leaves[3].grad)
    base, step = [x.double(), w.double(), b.double()], 1e-5
    for which in range(3):
        for i in range(0, base[which].numel(), 5):
            up, down = [v.clone() for v in base], [v.clone() for v in base]
            up[which].view(-1)[i] += step
            down[which].view(-1)[i] -= step
            g = float(leaves[which].grad.reshape(-1)[i])
            # differences: O(step^2) and the float64 sum's rounding over the step; the gradient itself float32
            assert abs((loss(*up) - loss(*down)) / (2 * step) - g) <= 2e-5 * (1 + abs(g))
    # a sum that nothing uses, a y that nothing uses, no shift
    xr, wr, br = (t.clone().requires_grad_(True) for t in (x, w, b))
    _, h = whtmix.LayerNormFunction.apply(xr, wr, br, r)
    (h * dh).sum().backward()
    assert torch.equal(xr.grad, dh) and bool((wr.grad == 0).all()) and bool((br.grad == 0).all()) and wr.grad.data_ptr() != br.grad.data_ptr()
    xr = x.clone().requires_grad_(True)
    y, _ = whtmix.LayerNormFunction.apply(xr, w)
    (g,) = torch.autograd.grad(y, xr, dy, create_graph=True)
    with pytest.raises(RuntimeError):
        g.sum().backward()


# ---- the gated half ----

def phi(z, act):
    """The activation and its derivative."""
    if act == "none":
        return z, torch.ones_like(z)
    if act == "relu":
        return z.clamp_min(0), (z > 0).double()
    c = math.sqrt(2.0 / math.pi)
    u, du = (z, 1.0) if act == "silu" else (2 * c * (z + 0.044715 * z ** 3), 2 * c * (1 + 3 * 0.044715 * z ** 2))
    s = torch.sigmoid(u)
    return z * s, s + z * s * torch.sigmoid(-u) * du


GATED_SHAPES = [  # T, N, K
    (1, 1, 1), (1, 64, 64), (1, 2736, 1024), (2, 427, 120), (7, 3, 5), (8, 777, 1003), (16, 130, 96), (17, 1000, 2048), (31, 1, 4000),
    (33, 513, 65), (64, 3000, 520), (65, 1000, 512), (100, 1024, 256), (127, 77, 1001), (128, 128, 128), (129, 256, 64), (200, 300, 256),
    (250, 512, 4096), (256, 512, 1024), (1000, 777, 1003), (129, 65, 40), (3000, 128, 512), (5000, 344, 128), (70, 4100, 264), (4097, 96, 81),
    (300, 8, 16), (20011, 152, 136), (2000, 129, 2000),
]


def check_gated(T, N, K, act, bias, eight, out_dtype, preact):
    x, w = rand(1, T, K), rand(2, 2 * N, K) / math.sqrt(K)
    kw = {}
    if eight:
        x, xs = whtmix.quantize_rows(x)
        w, ws = whtmix.quantize_rows(w)
        kw = {"x_scale": xs, "w_scale": ws}
        X, W = x.double() * xs.double()[:, None], w.double() * ws.double()[:, None]
    else:
        x, w = x.to(BF), w.to(BF)
        X, W = x.double(), w.double()
    b = rand(3, 2 * N) if bias else None
    out, out_ok = guarded((T, N), out_dtype)
    p_out, p_ok = guarded((T, 2 * N), BF) if preact else (None, lambda: None)
    got = whtmix.gated_linear(x, w, b, act, out_dtype=out_dtype, out=out, preact=p_out, **kw)
    assert (got[0] if preact else got) is out
    out_ok()
    p_ok()
    p = X @ W.T + (b.double() if bias else 0.0)
    p_err = K * 2.0 ** -23 * (X.abs() @ W.abs().T) + 8 * U32 * p.abs()
    (g, u), (g_err, u_err) = p.split(N, 1), p_err.split(N, 1)
    a, slope = phi(g, act)
    a_err = 1.2 * g_err + 2.0 ** -17 * a.abs() + 2.0 ** -17 * (g * slope).abs()  # every |slope| <= 1.13
    y = a * u
    y_err = a_err * (u.abs() + u_err) + a.abs() * u_err + U32 * y.abs()
    close(out, y, rounded(y, y_err, out_dtype))
    if preact:
        close(p_out, p, rounded(p, p_err, BF))
    plain = whtmix.gated_linear(x, w, b, act, out_dtype=out_dtype, preact=preact, **kw)  # the compiled way
    assert torch.equal(plain[0] if preact else plain, out) and (not preact or torch.equal(plain[1], p_out))


@pytest.mark.parametrize("T,N,K", GATED_SHAPES)
def test_gated_against_float64(T, N, K):
    check_gated(T, N, K, "silu", True, False, BF, False)
    check_gated(T, N, K, "gelu", True, False, BF, True)
    check_gated(T, N, K, "relu", False, False, F32, False)
    check_gated(T, N, K, "none", False, False, BF, True)


@pytest.mark.parametrize("T,N,K", GATED_SHAPES)
def test_eight_bit_gated_against_float64(T, N, K):
    check_gated(T, N, K, "silu", True, True, BF, True)
    check_gated(T, N, K, "gelu", False, True, F32, False)


@pytest.mark.parametrize("T,N,K", [(8192, 2048, 1024), (5000, 2100, 2000), (9001, 1024, 1003), (40000, 264, 64)])
def test_large_gated_against_float64(T, N, K):
    """Two CTAs on a tile, several tiles a CTA; the last tiles of rows and columns cut."""
    check_gated(T, N, K, "gelu", True, False, BF, True)
    check_gated(T, N, K, "silu", True, True, F32, False)


def test_gated_of_integers_is_exact():
    """Small integers: g and u are exact in float32, y is their product rounded once: one wrong element shows."""
    g = torch.Generator(device="cuda")
    g.manual_seed(7)
    for T, N, K in [(1, 300, 200), (50, 129, 77), (120, 256, 1024), (300, 777, 333), (2000, 520, 128), (8000, 2048, 1500)]:
        x = torch.randint(-3, 4, (T, K), generator=g, device="cuda").to(BF)
        w = torch.randint(-3, 4, (2 * N, K), generator=g, device="cuda").to(BF)
        b = torch.randint(-9, 10, (2 * N,), generator=g, device="cuda").float()
        p = x.double() @ w.double().T + b.double()
        for act in ("none", "relu"):
            want = phi(p[:, :N], act)[0] * p[:, N:]
            assert torch.equal(whtmix.gated_linear(x, w, b, act, out_dtype=F32), want.float())
        ones_x, ones_w = torch.ones(T, device="cuda"), torch.full((2 * N,), 2.0, device="cuda")
        y8 = whtmix.gated_linear(x.to(E4M3), w.to(E4M3), None, "none", x_scale=ones_x, w_scale=ones_w, out_dtype=F32)
        q = 2 * (x.double() @ w.double().T)
        assert torch.equal(y8, (q[:, :N] * q[:, N:]).float())
        # dp = [dy u, dy g] of small integers is exact in bf16
        dy = torch.randint(-3, 4, (T, N), generator=g, device="cuda").to(BF)
        pi = torch.randint(-9, 10, (T, 2 * N), generator=g, device="cuda").to(BF)
        _, dw, db = whtmix.gated_linear_backward(x, w, dy, pi, "none", dw_dtype=F32)
        dp = torch.cat([dy.double() * pi[:, N:].double(), dy.double() * pi[:, :N].double()], 1)
        assert torch.equal(dw.double(), dp.T @ x.double()) and torch.equal(db.double(), dp.sum(0))


def test_gated_strided_misaligned_and_between_rows():
    """Rows at other pitches and alignments; the elements between them are someone else's: neither read nor written."""
    for T in (1, 9, 200, 700):
        for K, N in ((300, 129), (67, 1002), (128, 68), (192, 256)):
            kp, np_ = (K + 7) // 8 * 8 + 8, (2 * N + 7) // 8 * 8 + 8
            x, w = torch.full((T, kp), math.nan, device="cuda").to(BF), torch.full((2 * N, kp), math.nan, device="cuda").to(BF)
            x[:, :K], w[:, :K] = rand(1, T, K).to(BF), (rand(2, 2 * N, K) / math.sqrt(K)).to(BF)
            b = rand(3, 2 * N)
            y, p = (torch.full((T, np_), 7.0, device="cuda").to(BF) for _ in range(2))
            whtmix.gated_linear(x[:, :K], w[:, :K], b, "gelu", preact=p[:, :2 * N], out=y[:, :N])
            want, want_p = whtmix.gated_linear(x[:, :K].contiguous(), w[:, :K].contiguous(), b, "gelu", preact=True)
            assert torch.equal(y[:, :N], want) and bool((y[:, N:] == 7).all())
            assert torch.equal(p[:, :2 * N], want_p) and bool((p[:, 2 * N:] == 7).all())
            y.fill_(7.0), p.fill_(7.0)
            whtmix.gated_linear(x[:, :K], w[:, :K], b, "gelu", preact=p[:, 3:2 * N + 3], out=y[:, 1:N + 1])  # any two-byte address
            assert torch.equal(y[:, 1:N + 1], want) and bool((y[:, 0] == 7).all()) and bool((y[:, N + 1:] == 7).all())
            assert torch.equal(p[:, 3:2 * N + 3], want_p) and bool((p[:, :3] == 7).all()) and bool((p[:, 2 * N + 3:] == 7).all())
            dy = torch.full((T, np_), math.nan, device="cuda").to(BF)
            dy[:, :N] = rand(4, T, N).to(BF)
            dx = torch.full((T, kp), 7.0, device="cuda").to(BF)
            got = whtmix.gated_linear_backward(x[:, :K], w[:, :K], dy[:, :N], p[:, 3:2 * N + 3], "gelu", dx=dx[:, :K])
            want = whtmix.gated_linear_backward(x[:, :K].contiguous(), w[:, :K].contiguous(), dy[:, :N].contiguous(), want_p, "gelu")
            assert bool((dx[:, K:] == 7).all()) and all(torch.equal(s, t) for s, t in zip(got, want))
    # three leading axes, and every second token
    x, w = rand(1, 40, 96).to(BF), (rand(2, 160, 96) / 10).to(BF)
    y = whtmix.gated_linear(x, w)
    assert torch.equal(whtmix.gated_linear(x.view(2, 4, 5, 96), w), y.view(2, 4, 5, 80))
    close(whtmix.gated_linear(x[::2], w), y[::2].double(), 2 * U16 * y[::2].double().abs() + 2.0 ** -12)


def test_values_that_are_not_finite_stay_where_they_are():
    """An infinity or a NaN in one token or one channel reaches that row or column only, and no neighbour in an epilogue."""
    N, K = 200, 96
    w, b = (rand(2, 2 * N, K) / 10).to(BF), rand(3, 2 * N)
    for T in (150, 20):
        x, dy = rand(1, T, K).to(BF), rand(4, T, N).to(BF)
        for act in ACTS:
            clean, p = whtmix.gated_linear(x, w, b, act, preact=True)
            bad = x.clone()
            bad[7, 5], bad[9, 1] = math.nan, math.inf
            rest = [i for i in range(T) if i not in (7, 9)]
            got = whtmix.gated_linear(bad, w, b, act)
            assert bool(torch.isnan(got[7]).all()) and torch.equal(got[rest], clean[rest])
            cols = [i for i in range(N) if i != 11]
            for place in (11, N + 11):  # in the gate, in the value
                ww = w.clone()
                ww[place, 3] = math.nan
                got = whtmix.gated_linear(x, ww, b, act)
                assert bool(torch.isnan(got[:, 11]).all()) and torch.equal(got[:, cols], clean[:, cols])
                pp = p.clone()
                pp[5, place] = math.nan
                grads, ref = whtmix.gated_linear_backward(x, w, dy, pp, act), whtmix.gated_linear_backward(x, w, dy, p, act)
                others = [i for i in range(T) if i != 5]
                assert bool(torch.isnan(grads[0][5]).all()) and torch.equal(grads[0][others], ref[0][others])
                rows = [i for i in range(2 * N) if i not in (11, N + 11)]
                assert torch.equal(grads[1][rows], ref[1][rows]) and torch.equal(grads[2][rows], ref[2][rows])
                assert bool(torch.isnan(grads[2][[11, N + 11]]).any())
    # far ends of the gate
    z = torch.tensor([-3.0e38, -1.0e30, -1e4, -88.0, -40.0, 0.0, 40.0, 1e4, 1e30, 3e38], device="cuda")
    n = len(z)
    x1, w1 = torch.zeros(1, 8, device="cuda").to(BF), torch.zeros(2 * n, 8, device="cuda").to(BF)
    for act in ("gelu", "silu"):
        y = whtmix.gated_linear(x1, w1, torch.cat([z, torch.full_like(z, 0.5)]), act, out_dtype=F32)[0].double()
        close(y, 0.5 * phi(z.double(), act)[0], 2.0 ** -17 * z.double().clamp_min(0) + 1e-15)
        p = torch.cat([z, torch.full_like(z, 2.0)])[None].to(BF)
        _, _, db = whtmix.gated_linear_backward(x1, w1, torch.ones(1, n, device="cuda").to(BF), p, act)
        zb = z.to(BF).double()
        value, slope = phi(zb, act)
        slope = torch.where(zb.abs() > 1e20, (zb > 0).double(), slope)  # (z^3 overflows what z's slope has long reached)
        close(db, torch.cat([2 * slope, value]), torch.cat([2.0 ** -15 * torch.ones_like(z).double(), 2.0 ** -16 * zb.clamp_min(0) + 1e-15]))


def check_gated_backward(T, N, K, act, dw_dtype=BF, **need):
    x, w = rand(1, T, K).to(BF), (rand(2, 2 * N, K) / math.sqrt(K)).to(BF)
    dy, p = rand(3, T, N).to(BF), rand(4, T, 2 * N).to(BF)
    outs = [guarded((T, K), BF), guarded((2 * N, K), dw_dtype), guarded((2 * N,), F32)]
    given = {name: o for name, (o, _) in zip(("dx", "dw", "db"), outs) if need.get("need_" + name, True)}
    dx, dw, db = whtmix.gated_linear_backward(x, w, dy, p, act, dw_dtype=dw_dtype, **given, **need)
    for _, ok in outs:
        ok()
    D, (g, u) = dy.double(), p.double().split(N, 1)
    value, slope = phi(g, act)
    dp = torch.cat([D * u * slope, D * value], 1)
    exact = act in ("none", "relu")
    dp_err = 2 * U32 * dp.abs() if exact else torch.cat([2.0 ** -16 * (D * u).abs(), 2.0 ** -16 * (D * g).abs()], 1)
    if db is not None:
        close(db, dp.sum(0), (T / 16 + 100) * U32 * dp.abs().sum(0) + dp_err.sum(0) + 1e-30)
    term = U16 * dp.abs() + dp_err  # dp rounded once
    for got, a, b_, e in ((dx, dp, w.double(), term), (dw, dp.T, x.double(), term.T)):
        if got is None:
            continue
        ref = a @ b_
        err = e @ b_.abs() + a.shape[1] * 2.0 ** -23 * (a.abs() @ b_.abs())
        close(got, ref, rounded(ref, err, got.dtype) + 1e-30)
        # and as a whole: roundings of random sign
        assert float((got.double() - ref).norm()) <= 2 * U16 * float(ref.norm()) + 1e-30
    again = whtmix.gated_linear_backward(x, w, dy, p, act, dw_dtype=dw_dtype, **need)  # the compiled way; a fixed order of additions
    for s, t, name in zip(again, (dx, dw, db), ("dx", "dw", "db")):
        assert torch.equal(s, t) if need.get("need_" + name, True) else s is None and t is None
    return x, w, dy, p, (dx, dw, db)


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("T,N,K", [(1, 1, 1), (1, 200, 300), (2, 427, 120), (20, 65, 33), (130, 64, 64), (136, 495, 928), (300, 130, 257),
                                   (1000, 256, 128), (2049, 96, 640), (5000, 344, 72), (4000, 33, 1000), (3001, 777, 1003)])
def test_gated_backward_against_float64(T, N, K, act):
    check_gated_backward(T, N, K, act)
    check_gated_backward(T, N, K, act, dw_dtype=F32)


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("T,N,K", [(9729, 688, 256), (12000, 200, 130), (20001, 72, 64), (10240, 264, 33), (9730, 100, 200), (8192, 1024, 2048)])
def test_gated_backward_of_many_tokens(T, N, K, act):
    x, w, dy, p, (dx, dw, db) = check_gated_backward(T, N, K, act)
    one = whtmix.gated_linear_backward(x, w, dy, p, act, need_dw=False, need_db=False)
    assert torch.equal(one[0], dx) and one[1] is None and one[2] is None
    # without dx another kernel makes dp: its float32 values may differ in their last bit, the bounds are the same
    check_gated_backward(T, N, K, act, need_dx=False)
    check_gated_backward(T, N, K, act, need_dx=False, need_dw=False)
    check_gated_backward(T, N, K, act, need_dx=False, need_db=False)


@pytest.mark.parametrize("T,N,K", [(9601, 64, 40), (9700, 8, 256), (9729, 6400, 64), (10001, 136, 129), (20000, 1000, 100), (9601, 9728, 8)])
def test_gated_backward_of_many_tokens_and_its_weight_gradient(T, N, K):
    check_gated_backward(T, N, K, "silu")
    check_gated_backward(T, N, K, "gelu", dw_dtype=F32, need_db=False)
    check_gated_backward(T, N, K, "relu", need_dw=False)


@pytest.mark.parametrize("T,N,K", [(8200, 1001, 40), (62000, 130, 24), (76000, 101, 16), (120000, 57, 33), (6000, 1600, 300), (64, 1408, 96), (127, 149, 33)])
def test_gated_backward_of_rows_in_a_ring(T, N, K):
    """Enough rows a thread for them to come through shared memory, each number of threads a row; rows that start anywhere between others'
    values, the first one inside its granule."""
    x, w, dy, p, want = check_gated_backward(T, N, K, "silu")
    if N % 8 == 0:
        return
    for offset, gap in ((1, 3), (5, 0), (7, 8)):
        buffers = [torch.full((T * (n + gap) + 16,), math.nan, device="cuda").to(BF) for n in (N, 2 * N)]
        dy2, p2 = (b[offset:offset + T * (n + gap)].view(T, n + gap)[:, :n] for b, n in zip(buffers, (N, 2 * N)))
        dy2.copy_(dy)
        p2.copy_(p)
        got = whtmix.gated_linear_backward(x, w, dy2, p2, "silu")
        assert all(torch.equal(s, t) for s, t in zip(got, want))


def test_gated_gradients_by_differences():
    """Against central differences of the float64 definition, through autograd; values that bf16 holds, small sizes."""
    T, N, K = 4, 12, 24
    x, w, b, dy = rand(1, T, K).to(BF), (rand(2, 2 * N, K) / 5).to(BF), rand(3, 2 * N), rand(5, T, N).to(BF)

    def loss(x_, w_, b_, act):
        p = x_ @ w_.T + b_
        return float((phi(p[:, :N], act)[0] * p[:, N:] * dy.double()).sum())

    for act in ACTS:
        leaves = [t.clone().requires_grad_(True) for t in (x, w, b)]
        y = whtmix.GatedLinearFunction.apply(*leaves, act)
        (y.float() * dy.float()).sum().backward()
        base, step = [x.double(), w.double(), b.double()], 1e-5
        for which in range(3):
            grad = leaves[which].grad.double()
            # p is stored in bf16 (2^-9 of g and of u, factors of one another), dp rounded, the result rounded
            tol = 10 * U16 * float(grad.abs().max()) + 1e-4
            for i in range(0, base[which].numel(), 7):
                up, down = [v.clone() for v in base], [v.clone() for v in base]
                up[which].view(-1)[i] += step
                down[which].view(-1)[i] -= step
                diff = (loss(*up, act) - loss(*down, act)) / (2 * step)
                if act == "relu" and abs(diff - float(grad.reshape(-1)[i])) > tol:
                    continue  # a kink between the two sides, or between g and its bf16
                assert abs(diff - float(grad.reshape(-1)[i])) <= tol
    w.requires_grad_(True)
    y = whtmix.GatedLinearFunction.apply(x, w)  # neither x nor a bias asks for a gradient
    (dw,) = torch.autograd.grad(y, w, dy)
    assert torch.equal(dw, whtmix.gated_linear_backward(x, w.detach(), dy, whtmix.gated_linear(x, w.detach(), preact=True)[1], need_dx=False)[1])


# ---- clipping ----

def norm_of(tensors):
    return math.sqrt(sum(float(t.double().square().sum()) for t in tensors))


def check_clip(tensors, max_norm, in_place=False):
    before = [t.clone() for t in tensors]
    norm64 = norm_of(before)
    got_norm = whtmix.global_norm(tensors)
    assert got_norm.shape == () and got_norm.dtype == F32
    assert abs(float(got_norm) - norm64) <= 36 * U32 * norm64
    outs = tensors if in_place else [guarded(tuple(t.shape), t.dtype) if t.is_contiguous() else (torch.empty_like(t), lambda: None) for t in tensors]
    given = tensors if in_place else [o for o, _ in outs]
    clipped, norm = whtmix.clip_by_global_norm(tensors, max_norm, out=given)
    assert float(norm) == float(got_norm) and len(clipped) == len(tensors) and all(a is b for a, b in zip(clipped, given))
    factor = min(1.0, max_norm / (norm64 + 1e-6))
    for t, was, c in zip(tensors, before, clipped):
        ref = was.double() * factor
        close(c, ref, rounded(ref, 40 * U32 * ref.abs(), t.dtype))
        if factor == 1.0:
            assert torch.equal(c, was)
        if not in_place:
            assert torch.equal(t, was)
    if not in_place:
        for _, ok in outs:
            ok()
        again, norm2 = whtmix.clip_by_global_norm(tensors, max_norm)
        assert float(norm2) == float(norm) and all(torch.equal(a, b) for a, b in zip(again, clipped))
    return clipped


@pytest.mark.parametrize("sizes", [[1], [7], [8], [1, 2, 3, 4, 5], [4096, 8192, 16384], [100003, 5, 64 * 1024, 31], [1 << 22, 3, (1 << 20) + 1],
                                   list(range(1, 64)), [17] * 65, [5000] * 600, [3] * 2000])
def test_clipping_against_float64(sizes):
    tensors = [rand(i, n).to(BF if i % 3 == 1 else F32) for i, n in enumerate(sizes)]
    for max_norm in (0.25, 1e9, 0.0):
        check_clip(tensors, max_norm)
    check_clip(tensors, 0.5, in_place=True)


def test_clipping_of_shapes_strides_and_empty_tensors():
    a, b = rand(1, 33, 65), rand(2, 3, 4, 5, 6).to(BF)
    tensors = [a.t(), b.permute(2, 0, 3, 1), torch.empty(0, 7, device="cuda"), rand(3, 1).reshape(()), rand(4, 1, 9)[:, ::1], a[:0]]
    clipped = check_clip([t for t in tensors], 0.125)
    assert clipped[0].shape == (65, 33)
    flat = rand(5, 1001)
    for start in (1, 2, 3, 5):  # any element-aligned address, in and out differing
        x = flat[start:start + 700]
        out = torch.full((710,), 7.0, device="cuda")
        whtmix.clip_by_global_norm([x], 0.5, out=[out[4 - start % 4:704 - start % 4]])
        ref = x.double() * min(1.0, 0.5 / (norm_of([x]) + 1e-6))
        close(out[4 - start % 4:704 - start % 4], ref, 41 * U32 * ref.abs())
        assert bool((out[:4 - start % 4] == 7).all()) and bool((out[704 - start % 4:] == 7).all())
        y = flat.to(BF)[start:start + 700]
        check_clip([y, x], 0.5)
    assert float(whtmix.global_norm([torch.empty(0, device="cuda")])) == 0.0
    out, norm = whtmix.clip_by_global_norm([torch.empty(0, device="cuda")], 1.0)
    assert float(norm) == 0.0 and out[0].shape == (0,)
    same = rand(6, 100)
    assert abs(float(whtmix.global_norm([same, same])) - math.sqrt(2) * norm_of([same])) <= 40 * U32 * 2 * norm_of([same])


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("size", [1e-42, 1e-38, 1e-30, 1e-22, 1e-16, 1e17, 1e19, 1e30, 1e38])
def test_norms_whose_squares_leave_float32(size, dtype):
    """Values of any size have their norm: the float32 squares alone would be 0 or infinite."""
    t = (rand(1, 5000).clamp(-3, 3) * size).to(dtype)
    zeros = torch.zeros(70000, device="cuda")
    n = norm_of([t])
    got = float(whtmix.global_norm([t, zeros]))
    largest = float(torch.finfo(F32).max)  # a norm beyond it is infinite as a float32 (its factor comes from the float64 one)
    assert abs(got - n) <= 40 * U32 * n + 2.0 ** -149 if n <= largest else got == math.inf
    mixed = [t, rand(2, 100) * math.sqrt(max(size, 1e-30))]
    n = norm_of(mixed)
    got = float(whtmix.global_norm(mixed))
    assert abs(got - n) <= 40 * U32 * n + 2.0 ** -149 if n <= largest else got == math.inf
    out, _ = whtmix.clip_by_global_norm([t], 1.0)
    ref = t.double() * min(1.0, 1.0 / (norm_of([t]) + 1e-6))
    close(out[0], ref, rounded(ref, 42 * U32 * ref.abs(), dtype) + (2.0 ** -133 if dtype == BF else 2.0 ** -149))


def test_lists_that_are_not_finite():
    a, b = rand(1, 3000), rand(2, 500).to(BF)
    a[17] = math.inf
    out, norm = whtmix.clip_by_global_norm([a, b], 1.0)
    assert math.isinf(float(norm))
    assert bool(torch.isnan(out[0][17])) and bool((out[0][:17] == 0).all()) and bool((out[1] == 0).all())
    a[18] = math.nan
    out, norm = whtmix.clip_by_global_norm([a, b], 1.0, out=[a, b])
    assert math.isnan(float(norm)) and bool(torch.isnan(b).all())
    out, _ = whtmix.clip_by_global_norm([rand(3, 10)], math.inf)
    assert torch.equal(out[0], rand(3, 10))


# ---- together, on streams and in graphs ----

def feed_forward(x, r, gain, shift, w1, b1, w2, dy, stream=None):
    """The second half of a layer and its gradients, clipped."""
    y, h = whtmix.layer_norm(x, gain, shift, residual=r, stream=stream)
    z, p = whtmix.gated_linear(y, w1, b1, "silu", preact=True, stream=stream)
    o = whtmix.linear(z, w2, residual=h, stream=stream)
    dz, dw2, db2 = whtmix.linear_backward(z, w2, dy, need_db=True, stream=stream)
    dn, dw1, db1 = whtmix.gated_linear_backward(y, w1, dz, p, "silu", stream=stream)
    dx, dg, ds = whtmix.layer_norm_backward(h, gain, dn, dh=dy, stream=stream)
    clipped, norm = whtmix.clip_by_global_norm([dw1, db1, dw2, db2, dg, ds], 0.5, stream=stream)
    return [o, dx, norm] + clipped


def feed_forward_inputs(T=300, K=200, N=168):
    return (rand(1, T, K).to(BF), rand(2, T, K).to(BF), 1.0 + 0.1 * rand(3, K), 0.1 * rand(4, K), (rand(5, 2 * N, K) / 14).to(BF), rand(6, 2 * N),
            (rand(7, K, N) / 13).to(BF), rand(8, T, K).to(BF))


def test_the_half_layer_against_float64():
    args = feed_forward_inputs()
    o, dx, norm, dw1, db1, dw2, db2, dg, ds = feed_forward(*args)
    x, r, gain, shift, w1, b1, w2, dy = (t.double() for t in args)
    leaves = [t.requires_grad_(True) for t in (x, gain, shift, w1, b1, w2)]
    h = x + r
    n = (h - h.mean(-1, keepdim=True)) / torch.sqrt(h.var(-1, keepdim=True, unbiased=False) + EPS) * gain + shift
    p = n @ w1.T + b1
    N = w1.shape[0] // 2
    ref = h + (p[:, :N] * torch.sigmoid(p[:, :N]) * p[:, N:]) @ w2.T
    (ref * dy).sum().backward()
    grads = [leaves[3].grad, leaves[4].grad, leaves[5].grad, dy.sum(0), leaves[1].grad, leaves[2].grad]
    want = math.sqrt(sum(float(g.square().sum()) for g in grads))
    # four or five bf16 roundings on the way (2^-8 each at most): the bf16 tolerance 1e-2 in the 2-norm, 2e-2 through the backward
    assert float((o.double() - ref).norm() / ref.norm()) <= 1e-2
    assert float((dx.double() - leaves[0].grad).norm() / leaves[0].grad.norm()) <= 2e-2
    assert abs(float(norm) - want) <= 1e-2 * want
    for got, g in zip((dw1, db1, dw2, db2, dg, ds), grads):
        assert float((got.double() - g * (0.5 / want)).norm()) <= 3e-2 * float(g.norm()) * 0.5 / want


def test_on_another_stream_and_in_graphs():
    args = feed_forward_inputs()
    want = feed_forward(*args)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got = feed_forward(*args)
    whtmix.sync(s)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    got = feed_forward(*args, stream=s)
    whtmix.sync(s)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        got = feed_forward(*args)
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def new_calls(x, gain, shift, w, b, dy, tensors):
    y = whtmix.layer_norm(x, gain, shift)
    z, p = whtmix.gated_linear(y, w, b, "gelu", preact=True)
    grads = whtmix.gated_linear_backward(y, w, dy, p, "gelu")
    dx = whtmix.layer_norm_backward(x, gain, grads[0])
    clipped, norm = whtmix.clip_by_global_norm(tensors, 0.5)
    return [y, z, p, *grads, *dx, norm, whtmix.global_norm(tensors), *clipped]


def test_graphs_captured_one_after_another_share_nothing():
    """Two graphs captured on one stream that no eager call has used, of different sizes, replayed at the same time on two streams and
    after larger eager calls: what each needs in between is its own."""
    inputs = []
    for i, (T, K, N) in enumerate([(2000, 135, 77), (3001, 203, 150)]):
        inputs.append((rand(i, T, K).to(BF), 1 + 0.1 * rand(20 + i, K), 0.1 * rand(30 + i, K), (rand(40 + i, 2 * N, K) / 12).to(BF), rand(50 + i, 2 * N),
                       rand(60 + i, T, N).to(BF), [rand(70 + i, 50000 + i), rand(80 + i, 333).to(BF)]))
    want = [[t.clone() for t in new_calls(*a)] for a in inputs]
    whtmix.release_workspaces()
    s = torch.cuda.Stream()
    graphs, outs = [], []
    for a in inputs:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            outs.append(new_calls(*a))
        graphs.append(g)
    one, two = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(20):
        with torch.cuda.stream(one):
            graphs[1].replay()
        with torch.cuda.stream(two):
            graphs[0].replay()
    torch.cuda.synchronize()
    for got, ref in zip(outs, want):
        assert all(torch.equal(a, b) for a, b in zip(got, ref))
    with torch.cuda.stream(s):  # eager calls on the stream of the capture
        big = new_calls(rand(1, 9000, 201).to(BF), 1 + 0.1 * rand(2, 201), rand(3, 201), (rand(4, 400, 201) / 14).to(BF), rand(5, 400),
                        rand(6, 9000, 200).to(BF), [rand(7, 1 << 21)])
    torch.cuda.synchronize()
    del big
    whtmix.release_workspaces()
    for got in outs:
        for t in got:
            t.zero_()
    graphs[0].replay()
    graphs[1].replay()
    torch.cuda.synchronize()
    for got, ref in zip(outs, want):
        assert all(torch.equal(a, b) for a, b in zip(got, ref))
    del graphs[0]
    graphs[0].replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs[1], want[1]))
    whtmix.sync(s)


def test_two_threads_on_one_stream():
    import threading
    s = torch.cuda.Stream()
    cases = []
    for i, T in enumerate((300, 5000)):
        h, w, dy = rand(i, T, 130).to(BF), 1 + 0.1 * rand(9, 130), rand(10 + i, T, 130).to(BF)
        cases.append((h, w, dy, whtmix.layer_norm_backward(h, w, dy)))
    torch.cuda.synchronize()
    wrong = []

    def work(case):
        h, w, dy, want = case
        torch.cuda.set_device(0)
        with torch.cuda.stream(s):
            for _ in range(200):
                got = whtmix.layer_norm_backward(h, w, dy)
                got_norm = whtmix.global_norm([h, dy])
            s.synchronize()
            if not all(torch.equal(a, b) for a, b in zip(got, want)) or abs(float(got_norm) - norm_of([h, dy])) > 1e-4 * float(got_norm):
                wrong.append(h.shape)

    threads = [threading.Thread(target=work, args=(c,)) for c in cases]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong


def test_two_threads_on_their_default_streams():
    """cudaStreamPerThread is one handle (2) for a stream of each host thread: their calls run at the same time."""
    import ctypes
    import threading
    lib = whtmix.library()
    cases = []
    for i, T in enumerate((4000, 5000)):
        h, w, dy = rand(i, T, 130).to(BF), 1 + 0.1 * rand(9, 130), rand(10 + i, T, 130).to(BF)
        cases.append((h, w, dy, whtmix.layer_norm_backward(h, w, dy), [torch.empty_like(h), torch.empty_like(w), torch.empty_like(w)]))
    torch.cuda.synchronize()
    codes = []

    def work(case):
        h, w, dy, _, (dx, dw, db) = case
        torch.cuda.set_device(0)
        for _ in range(100):
            codes.append(lib.whtmix_layer_norm_backward(h.data_ptr(), w.data_ptr(), dy.data_ptr(), None, dx.data_ptr(), dw.data_ptr(), db.data_ptr(),
                                                        *h.shape, 130, 130, 0, 130, 1e-5, 1, ctypes.c_void_p(2)))

    threads = [threading.Thread(target=work, args=(c,)) for c in cases]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert codes == [0] * 200
    for case in cases:
        assert all(torch.equal(a, b) for a, b in zip(case[4], case[3]))


FIRST_CALLS_IN_A_GRAPH = """
import torch
from paper_2607_25234_gb300 import whtmix
x, w = torch.randn(5000, 77, device="cuda"), torch.ones(77, device="cuda")
xb, wb = torch.randn(3000, 100, device="cuda").bfloat16(), torch.randn(120, 100, device="cuda").bfloat16()
def calls():
    dx = whtmix.layer_norm_backward(x, w, x)
    y, p = whtmix.gated_linear(xb, wb, preact=True)
    return [whtmix.layer_norm(x, w), *dx, y, p, *whtmix.gated_linear_backward(xb, wb, y, p), whtmix.global_norm([x, w])]
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    got = calls()
g.replay()
torch.cuda.synchronize()
assert all(torch.equal(a, b) for a, b in zip(got, calls()))
whtmix.sync()
print("the same")
"""


def test_a_processs_first_calls_may_be_captured():
    import os
    import subprocess
    import sys
    done = subprocess.run([sys.executable, "-c", FIRST_CALLS_IN_A_GRAPH], cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                          capture_output=True, text=True, timeout=300)
    assert done.returncode == 0 and "the same" in done.stdout, done.stderr[-2000:]


def test_a_backward_pass_in_a_graph():
    """Forward and backward captured after eager passes of the same leaves on another stream (whose autograd graphs are gone: torch joins
    the leaves' streams of a live one, which no capture allows, whatever the operators)."""
    x, w, b = rand(1, 64, 96).to(BF), (rand(2, 160, 96) / 10).to(BF).requires_grad_(True), rand(3, 160).requires_grad_(True)
    gain, shift = (1 + 0.1 * rand(4, 96)).requires_grad_(True), (0.1 * rand(5, 96)).requires_grad_(True)
    leaves = [w, b, gain, shift]

    def step():
        n, _ = whtmix.LayerNormFunction.apply(x, gain, shift)
        y = whtmix.GatedLinearFunction.apply(n, w, b, "gelu")
        return torch.autograd.grad(y, leaves, torch.ones_like(y))

    want = [g.clone() for g in step()]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        got = step()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b_) for a, b_ in zip(got, want))
    eager = step()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b_) for a, b_ in zip(eager, want)) and all(torch.equal(a, b_) for a, b_ in zip(got, want))


def test_nothing_to_do():
    w, gain, shift = (rand(2, 64, 32) / 5).to(BF), torch.ones(32, device="cuda"), torch.zeros(32, device="cuda")
    x = torch.empty(0, 32, dtype=BF, device="cuda")
    y, h = whtmix.layer_norm(x, gain, shift, residual=x)
    assert y.shape == (0, 32) and h.shape == (0, 32)
    q, s = whtmix.layer_norm(x, gain, out_dtype=E4M3)
    assert q.shape == (0, 32) and s.shape == (0,)
    y, p = whtmix.gated_linear(x, w, preact=True)
    assert y.shape == (0, 32) and p.shape == (0, 64)
    dx, dw, db = whtmix.layer_norm_backward(x, gain, x)
    assert dx.shape == (0, 32) and bool((dw == 0).all()) and bool((db == 0).all())
    dx, dw, db = whtmix.gated_linear_backward(x, w, torch.empty(0, 32, dtype=BF, device="cuda"), torch.empty(0, 64, dtype=BF, device="cuda"))
    assert dx.shape == (0, 32) and dw.shape == (64, 32) and bool((dw == 0).all()) and bool((db == 0).all())


def test_a_streams_first_call_may_be_the_smallest():
    x, w, dy = rand(1, 1, 1), torch.ones(1, device="cuda"), rand(2, 1, 1)
    whtmix.release_workspaces()
    check_norm_backward(x, w, dy, None)
    whtmix.release_workspaces()
    check_clip([rand(1, 1)], 0.5)
    whtmix.release_workspaces()
    check_gated(1, 1, 1, "silu", True, False, BF, True)
    check_gated_backward(3, 1, 5, "gelu")
    whtmix.sync()


def test_offsets_beyond_32_bits():
    """Rows and elements at more than 2^31 and 2^32: the first, one past each and the last are right."""
    T, D = (1 << 32) // 4096 + 70, 4096
    x = torch.zeros(T, D, dtype=BF, device="cuda")  # 8.6 GB
    rows = [0, (1 << 31) // D + 1, (1 << 32) // D + 3, T - 1]
    for i, t in enumerate(rows):
        x[t] = rand(i, D).to(BF)
    picked = x[rows]
    n = norm_of([picked])
    assert abs(float(whtmix.global_norm([x])) - n) <= 40 * U32 * n
    w = (rand(2, 128, D) / 64).to(BF)
    y, p = whtmix.gated_linear(x, w, None, "relu", preact=True)
    ref = picked.double() @ w.double().T
    size = D * 2.0 ** -23 * (picked.double().abs() @ w.double().abs().T)
    close(p[rows], ref, rounded(ref, size, BF))
    g, u = ref.split(64, 1)
    close(y[rows], g.clamp_min(0) * u, rounded(g.clamp_min(0) * u, size[:, :64] * (u.abs() + size[:, 64:]) + g.abs() * size[:, 64:], BF))
    assert float(p.float().abs().sum()) == float(p[rows].float().abs().sum())
    dy = torch.zeros(T, 64, dtype=BF, device="cuda")
    dy[rows] = rand(9, 4, 64).to(BF)
    dp = torch.cat([dy[rows].double() * p[rows][:, 64:].double() * (p[rows][:, :64] > 0), dy[rows].double() * p[rows][:, :64].double().clamp_min(0)], 1)
    _, dw, db = whtmix.gated_linear_backward(x, w, dy, p, "relu", need_dx=False, dw_dtype=F32)
    close(dw, dp.T @ picked.double(), (U16 + 2.0 ** -18) * (dp.abs().T @ picked.double().abs()) + 1e-30)
    del y, p
    gain, shift = torch.ones(D, device="cuda"), torch.zeros(D, device="cuda")
    ref, err = Norm(picked).y(gain, shift)
    out = whtmix.layer_norm(x, gain, shift, out=x)
    close(out[rows], ref, rounded(ref, err, BF))
    clipped, _ = whtmix.clip_by_global_norm([x], 1.0, out=[x])
    n = norm_of([out[rows]])
    assert abs(norm_of([clipped[0][rows]]) - 1.0) <= 2 * U16


# ---- the example ----

@pytest.fixture(scope="module")
def example():
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    spec = importlib.util.spec_from_file_location("mixer_layer", os.path.join(root, "examples", "mixer_layer.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def hadamard(n):
    h = torch.ones(1, 1, dtype=torch.float64, device="cuda")
    while h.shape[0] < n:
        h = torch.cat([torch.cat([h, h], 1), torch.cat([h, -h], 1)], 0)
    return h


def plain_layer(layer, x, params):
    """The layer in float64, without any of the library."""
    norm1, norm2, w_in, w_out, gains, w1, b1, w2, b2 = params[:9]
    shift1, shift2 = params[9:] if layer.norm == "layer" else (0.0, 0.0)
    N, C = gains.shape

    def norm(v, g, b):
        if layer.norm == "rms":
            return v * torch.rsqrt(v.square().mean(-1, keepdim=True) + 1e-6) * g
        return (v - v.mean(-1, keepdim=True)) * torch.rsqrt(v.var(-1, keepdim=True, unbiased=False) + EPS) * g + b

    HN, HC = hadamard(N), hadamard(C)
    z = norm(x, norm1, shift1) @ w_in.T
    h = x + (HN @ (gains * (HN @ z @ HC)) @ HC / (N * C)) @ w_out.T
    p = norm(h, norm2, shift2) @ w1.T + b1
    if layer.gated:
        hidden = w2.shape[1]
        u = p[..., :hidden] * torch.sigmoid(p[..., :hidden]) * p[..., hidden:]
    else:
        u = phi(p, "gelu")[0]
    return h + u @ w2.T + b2


@pytest.mark.parametrize("norm,gated", [("layer", True), ("layer", False), ("rms", True)])
@pytest.mark.parametrize("B,N,C", [(2, 256, 64), (1, 1024, 128)])
def test_the_example_with_layer_norm_and_gated_half(example, norm, gated, B, N, C):
    layer = example.MixerLayer(N, C, norm=norm, gated=gated)
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    params = layer.parameters()
    for p in params:
        if p.dtype == F32:
            p += 0.1 * torch.randn(p.shape, generator=g, device="cuda")
    x, dy = torch.randn(B, N, C, generator=g, device="cuda").to(BF), torch.randn(B, N, C, generator=g, device="cuda").to(BF)
    exact = [p.double().requires_grad_(True) for p in params]
    xe = x.double().requires_grad_(True)
    ye = plain_layer(layer, xe, exact)
    (ye * dy.double()).sum().backward()
    for p in params:
        p.requires_grad_(True)
    xr = x.clone().requires_grad_(True)
    y = layer.train_forward(xr)
    # about ten bf16 roundings of activations on the way, each 2^-8 of a value at most: the bf16 tolerance 1e-2 in the 2-norm
    assert float((y.detach().double() - ye.detach()).norm() / ye.detach().norm()) <= 1e-2
    (y.float() * dy.float()).sum().backward()
    for got, want in zip([xr] + params, [xe] + exact):
        assert float((got.grad.double() - want.grad).norm() / want.grad.norm()) <= 2e-2  # both ways' roundings together
    grads = [p.grad.clone() for p in params]
    n = norm_of(grads)
    clipped, _ = whtmix.clip_by_global_norm([p.grad for p in params], 0.5 * n, out=[p.grad for p in params])
    for p, before in zip(params, grads):
        close(p.grad, before.double() * 0.5, rounded(before.double() * 0.5, 40 * U32 * before.double().abs(), p.dtype))
        p.requires_grad_(False)
    out = layer.forward(x)
    assert torch.equal(out, y.detach())
    layer.quantize()
    # e4m3 rounds each activation and weight by 2^-5 of it on average at most: the first product's error is that, one half of y
    assert float((layer.forward(x).double() - ye.detach()).norm() / ye.detach().norm()) <= 6e-2
    losses = example.train(layer, x, dy.float(), 3, max_norm=1.0)
    assert len(losses) == 3 and all(math.isfinite(v) for v in losses)
    whtmix.sync()
