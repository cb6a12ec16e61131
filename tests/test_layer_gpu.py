"""The layer operators around the mixer on a GPU: RMS norm with the residual's addition (and its 8-bit output), the matrix
product with bias, activation and residual, and both backwards, against plain float64 implementations.

Tolerances, derived before any run.  u16 = 2^-8 is the most that rounding to bf16 (8 significand bits) moves a value by, relative
to it; u32 = 2^-24 is float32's.
  * a bf16 output is a value y32 rounded once: |got - ref| <= u16 |ref| (1 + u16) + the error of y32.
  * norm: y32 = h rstd w.  The row's sum of D squares of positive terms has a relative error of at most (D / 32 + 40) u32 (each
    thread adds at most D / 32 terms, then at most 16 partial sums and shuffles), half of which reaches rstd; rsqrt adds 2^-22;
    three more roundings.  D <= 2^14 here except where a case says otherwise: 2^-13.  For float32 a factor of 4 above the usual
    square-root growth, 2^-20, is held in the 2-norm, and the bound above element by element.
  * products: a sum of K terms in float32, the tensor cores' additions truncated: K 2^-23 (|x| |w|^T) element by element (K / 16
    additions of 16 products each, every one truncated by at most 2^-23 of the running sum, which |x| |w|^T bounds; the factor
    16 to spare covers the order inside a step and the scales).
  * activations: ex2 and rcp at 2^-22, their argument's rounding times the slope of the exponential (|u| <= 40: 2^-18): 2^-17
    |y| + 2^-17 |p slope| for the pre-activation's own error.
  * 8 bits: the values that a scale stands for are within half a step of the exact row (2^-4 of a value, 2^-10 of the row's
    largest below the smallest normal step); away from a tie they are the nearest, so that all but few are equal.
  * gradients: dp is rounded to bf16 before its products (u16 |dp| in each term), db and dw of the norm are float32 sums.
"""
import math

import pytest
import torch

from paper_2607_25234_gb300 import whtmix

pytestmark = pytest.mark.gpu

U16, U32 = 2.0 ** -8, 2.0 ** -24
BF, F32, E4M3 = torch.bfloat16, torch.float32, torch.float8_e4m3fn
EPS = 1e-6


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


def guarded(shape, dtype):
    """A view into a buffer with guard bytes around it, and a check that they are untouched."""
    n = math.prod(shape) * torch.empty((), dtype=dtype).element_size()
    buf = torch.full((n + 512,), 0x5A, dtype=torch.uint8, device="cuda")
    view = buf[256:256 + n].view(dtype).view(*shape)

    def check():
        assert bool((buf[:256] == 0x5A).all()) and bool((buf[256 + n:] == 0x5A).all()), "written outside the output"
    return view, check


# ---- RMS norm ----

def norm_ref(x, r, w, eps=EPS):
    h = x.double() if r is None else x.double() + r.double()
    rstd = 1.0 / torch.sqrt(h.square().mean(-1, keepdim=True) + eps)
    return h, h * rstd * w.double(), rstd


def e4m3_step(v):
    """The distance of e4m3 values around v: 2^(e - 3) for |v| in [2^e, 2^(e + 1)), e >= -6, exactly (the exponent's bits)."""
    bits = v.abs().clamp_min(2.0 ** -6).view(torch.int64)
    return ((bits >> 52) - 3 << 52).view(torch.float64)


def nearest_e4m3(v):
    """The e4m3 value nearest to v in float64, ties to even."""
    step = e4m3_step(v)
    return (torch.round(v / step) * step).clamp(-448.0, 448.0)


NORM_SHAPES = [(1, 1), (1, 8), (1, 256), (3, 7), (5, 64), (17, 65), (100, 128), (70, 100), (257, 512), (33, 1000), (64, 1024), (40, 2048),
               (12, 5001), (200, 5000), (7, 8192), (5, 16384), (400, 16), (300, 3000)]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T,D", NORM_SHAPES)
def test_norm_against_float64(T, D, dtype):
    w = 1.0 + 0.1 * rand(3, D)
    for residual in (False, True):
        x, r = rand(1, T, D).to(dtype), rand(2, T, D).to(dtype) if residual else None
        out, out_ok = guarded((T, D), dtype)
        h_out, h_ok = guarded((T, D), dtype) if residual else (None, lambda: None)
        before = x.clone()
        got = whtmix.rms_norm(x, w, residual=r, out=out, h=h_out)
        h, y, _ = norm_ref(x, r, w)
        unit = U16 if dtype == BF else U32
        y32 = (D / 32 + 60) * U32 * y.abs() + 2.0 ** -21 * y.abs()
        close(out, y, unit * (1 + U16) * y.abs() + y32 + 1e-37)
        if dtype == F32:
            assert float((out.double() - y).norm() / y.norm()) <= 2.0 ** -20
        out_ok()
        if residual:
            assert got[0] is out and got[1] is h_out
            close(h_out, h, (unit * (1 + U16) + U32) * h.abs() + 1e-37)
            h_ok()
        assert torch.equal(x, before)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T,D", NORM_SHAPES)
def test_norm_to_eight_bits(T, D, dtype):
    w = 1.0 + 0.1 * rand(3, D)
    x, r = rand(1, T, D).to(dtype), rand(2, T, D).to(dtype)
    q, scale, h32 = whtmix.rms_norm(x, w, residual=r, out_dtype=E4M3)
    assert q.dtype == E4M3 and q.shape == x.shape and scale.shape == (T,)
    _, y, _ = norm_ref(x, r, w)
    s = y.abs().amax(-1) / 448.0
    close(scale, s, ((D / 32 + 80) * U32 + 2.0 ** -20) * s)
    v = y / s[:, None]
    exact = nearest_e4m3(v)
    # a value may go to the other neighbour where it lies within rounding of the middle
    close(q.float(), v, e4m3_step(v) / 2 * (1 + 2.0 ** -12) + 2.0 ** -16 * v.abs())
    assert float((q.double() != exact).double().mean()) <= 1e-4 + 2.0 / v.numel()


@pytest.mark.parametrize("T,D", [(1, 1024), (3, 65), (2, 20001), (1, 100000)])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_norm_of_rows_beyond_the_registers_and_single_rows(T, D, dtype):
    w, x, r = 1.0 + 0.1 * rand(3, D), rand(1, T, D).to(dtype), rand(2, T, D).to(dtype)
    y, h = whtmix.rms_norm(x, w, residual=r)
    h_ref, ref, rstd = norm_ref(x, r, w)
    unit = U16 if dtype == BF else U32
    close(y, ref, (unit * (1 + U16) + (D / 32 + 60) * U32 + 2.0 ** -21) * ref.abs() + 1e-37)
    q, scale = whtmix.rms_norm(x, w, out_dtype=E4M3)
    ref0 = norm_ref(x, None, w)[1]
    close(q.double() * scale.double()[:, None], ref0, 2.0 ** -4 * (1 + 2.0 ** -8) * ref0.abs() + scale.double()[:, None] * 2.0 ** -9)
    dy = rand(4, T, D).to(dtype)
    check_norm_backward(h, w, dy, None)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_norm_in_place_and_strided(dtype):
    T, D = 65, 1000
    w, wide, r = 1.0 + 0.1 * rand(3, D), rand(1, T, 3 * D + 1).to(dtype), rand(2, T, D).to(dtype)
    for start in (0, 1, D + 1):  # aligned and not: the rows' distance is 3 D + 1 elements
        x = wide[:, start:start + D]
        y, h = whtmix.rms_norm(x, w, residual=r)
        plain = whtmix.rms_norm(x.contiguous(), w, residual=r)
        assert torch.equal(h, plain[1])
        ref = norm_ref(x, r, w)[1]
        close(y, ref, (U16 if dtype == BF else 2.0 ** -19) * 1.01 * ref.abs() + 2.0 ** -18 * ref.abs())
    x = rand(1, T, D).to(dtype)
    want_y, want_h = whtmix.rms_norm(x, w, residual=r)
    for target in ("x", "r"):
        a, b = x.clone(), r.clone()
        t = a if target == "x" else b
        y, h = whtmix.rms_norm(a, w, residual=b, h=t)
        assert h is t and torch.equal(h, want_h) and torch.equal(y, want_y)
    a = x.clone()
    assert torch.equal(whtmix.rms_norm(a, w, out=a), whtmix.rms_norm(x, w))
    views = rand(9, 6, 5, 4, 64).to(dtype)[::2, 1]  # [3, 4, 64], two strides
    with pytest.raises(ValueError, match="one stride"):
        whtmix.rms_norm(views, 1.0 + 0.1 * rand(3, 64))


@pytest.mark.parametrize("D", [128, 1001])
def test_norm_of_rows_that_are_empty_or_not_finite(D):
    w = torch.ones(D, device="cuda")
    x = rand(1, 6, D)
    x[0] = 0
    x[1, 3] = math.inf
    x[2, 5] = math.nan
    x[3] *= 1e-30
    x[4] *= 1e15
    x[5, 1:] = 0
    y = whtmix.rms_norm(x, w)
    ref = norm_ref(x, None, w)[1]
    assert bool((y[0] == 0).all())
    assert torch.isnan(y[1, 3]) and bool((y[1, :3] == 0).all()) and bool(torch.isnan(y[2]).all())
    close(y[[3, 4, 5]], ref[[3, 4, 5]], 2.0 ** -18 * ref[[3, 4, 5]].abs() + 1e-37)
    q, scale = whtmix.rms_norm(x, w, out_dtype=E4M3)
    assert float(scale[0]) == 0.0 and bool((q[0].float() == 0).all())
    assert torch.isnan(scale[1]) and torch.isnan(scale[2])
    for i in (3, 4, 5):
        top = float(ref[i].abs().max())
        close(q[i].double() * scale[i].double(), ref[i], 2.0 ** -4 * 1.01 * ref[i].abs() + top * 2.0 ** -17)
    # bf16, the type's largest and smallest values
    big = torch.full((1, D), 3.0e38, device="cuda").to(BF)
    tiny = torch.full((1, D), 1.0e-38, device="cuda").to(BF)
    assert bool((whtmix.rms_norm(big, w) == 0).all())  # the float32 sum of squares is infinite
    t = whtmix.rms_norm(tiny, w, eps=0.0)
    assert t.shape == tiny.shape


def check_norm_backward(h, w, dy, dh):
    dx_out, dx_ok = guarded(tuple(h.shape), h.dtype)
    dw_out, dw_ok = guarded((h.shape[-1],), F32)
    dx, dw = whtmix.rms_norm_backward(h, w, dy, dh=dh, dx=dx_out, dw=dw_out)
    dx_ok()
    dw_ok()
    D, T = h.shape[-1], h.shape[0]
    H, W, G = h.double(), w.double(), dy.double()
    rstd = 1.0 / torch.sqrt(H.square().mean(-1, keepdim=True) + EPS)
    a = G * W
    ref = rstd * a - H * rstd ** 3 * (a * H).mean(-1, keepdim=True)
    spread = rstd * a.abs() + H.abs() * rstd ** 3 * (a * H).abs().mean(-1, keepdim=True)
    if dh is not None:
        ref = ref + dh.double()
        spread = spread + dh.double().abs()
    unit = U16 if h.dtype == BF else U32
    close(dx, ref, unit * (1 + U16) * ref.abs() + ((D / 32 + 80) * U32 + 2.0 ** -19) * spread + 1e-37)
    n = H * rstd
    close(dw, (G * n).sum(0), ((T / 32 + D / 32 + 200) * U32 + 2.0 ** -19) * (G * n).abs().sum(0) + 1e-37)
    return dx, dw


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T,D", NORM_SHAPES + [(3001, 64), (1500, 257)])
def test_norm_backward_against_float64(T, D, dtype):
    w, h, dy, dh = 1.0 + 0.1 * rand(3, D), rand(1, T, D).to(dtype), rand(4, T, D).to(dtype), rand(5, T, D).to(dtype)
    check_norm_backward(h, w, dy, None)
    dx, dw = check_norm_backward(h, w, dy, dh)
    again = whtmix.rms_norm_backward(h, w, dy, dh=dh)
    assert torch.equal(dx, again[0]) and torch.equal(dw, again[1])  # a fixed order of additions
    for inplace in ("dy", "dh"):
        a, b = dy.clone(), dh.clone()
        got, _ = whtmix.rms_norm_backward(h, w, a, dh=b, dx=a if inplace == "dy" else b)
        assert torch.equal(got, dx)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T,D", [(1216, 177), (1217, 177), (5000, 9), (2433, 1001), (1300, 500), (620, 257), (3001, 77), (1219, 12), (1300, 1023),
                                 (20003, 33), (1223, 513), (1231, 5)])
def test_norm_of_many_odd_rows(T, D, dtype):
    """Contiguous rows that share their 16-byte pieces, both directions; also in place and beside a matrix that starts elsewhere."""
    test_norm_against_float64(T, D, dtype)
    w, h, dy, dh = 1.0 + 0.1 * rand(3, D), rand(1, T, D).to(dtype), rand(4, T, D).to(dtype), rand(5, T, D).to(dtype)
    check_norm_backward(h, w, dy, None)
    dx, dw = check_norm_backward(h, w, dy, dh)
    again = whtmix.rms_norm_backward(h, w, dy, dh=dh, dx=dy)
    assert torch.equal(again[0], dx) and torch.equal(again[1], dw)
    y, s = whtmix.rms_norm(h, w, residual=dh)
    x = h.clone()
    y2, s2 = whtmix.rms_norm(x, w, residual=dh, h=x)
    assert torch.equal(y, y2) and torch.equal(s, s2) and s2 is x
    shifted = torch.empty(T * D + 1, dtype=dtype, device="cuda")[1:].view(T, D).copy_(h)
    y3, _ = whtmix.rms_norm(shifted, w, residual=dh)
    close(y3, y.double(), 2 * (U16 if dtype == BF else (D / 32 + 200) * U32) * y.double().abs() + 1e-37)


def test_a_row_that_is_not_finite_leaves_its_neighbours():
    T, D = 2000, 177
    for dtype in (BF, F32):
        x, w, dy = rand(1, T, D).to(dtype), 1.0 + 0.1 * rand(3, D), rand(4, T, D).to(dtype)
        y, (dx, _) = whtmix.rms_norm(x, w), whtmix.rms_norm_backward(x, w, dy)
        bad = x.clone()
        bad[5, 7], bad[11, 0], bad[12, D - 1], bad[T - 1, 3] = float("nan"), float("inf"), float("nan"), float("nan")
        rows = torch.ones(T, dtype=torch.bool, device="cuda")
        rows[[5, 11, 12, T - 1]] = False
        y2, (dx2, dw2) = whtmix.rms_norm(bad, w), whtmix.rms_norm_backward(bad, w, dy)
        assert torch.equal(y[rows], y2[rows]) and torch.equal(dx[rows], dx2[rows])
        assert bool(torch.isnan(y2[5]).all()) and bool(torch.isnan(y2[12]).all()) and bool(torch.isnan(dw2).all())


def test_norm_gradients_by_differences():
    T, D = 3, 24
    x, r, w = rand(1, T, D), rand(2, T, D), 1.0 + 0.1 * rand(3, D)
    dy, dh = rand(4, T, D), rand(5, T, D)

    def loss(x_, w_):
        h, y, _ = norm_ref(x_, r, w_)
        return float((y * dy.double()).sum() + (h * dh.double()).sum())

    xr, wr, rr = x.clone().requires_grad_(True), w.clone().requires_grad_(True), r.clone().requires_grad_(True)
    y, h = whtmix.RMSNormFunction.apply(xr, wr, rr, EPS)
    ((y * dy).sum() + (h * dh).sum()).backward()
    assert torch.equal(xr.grad, rr.grad)
    step = 1e-5
    for t, grad, which in ((x, xr.grad, 0), (w, wr.grad, 1)):
        for i in range(0, t.numel(), 5):
            d = torch.zeros_like(t, dtype=torch.float64).view(-1)
            d[i] = step
            d = d.view(t.shape)
            up = loss(x.double() + d, w.double()) if which == 0 else loss(x.double(), w.double() + d)
            down = loss(x.double() - d, w.double()) if which == 0 else loss(x.double(), w.double() - d)
            # differences: O(step^2) and the float64 sum's rounding over the step; the gradient itself float32
            assert abs((up - down) / (2 * step) - float(grad.view(-1)[i])) <= 2e-5 * (1 + abs(float(grad.view(-1)[i])))


# ---- linear ----

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


LINEAR_SHAPES = [  # T, N, K
    (1, 1, 1), (1, 64, 64), (1, 4096, 1024), (2, 427, 120), (7, 3, 5), (8, 777, 1003), (16, 130, 96), (17, 1000, 2048), (31, 1, 4000),
    (33, 513, 65), (64, 3000, 520), (65, 1000, 512), (100, 1024, 256), (127, 77, 1001), (128, 128, 128), (129, 256, 64), (200, 300, 256),
    (250, 512, 4096), (256, 512, 1024), (1000, 777, 1003), (129, 65, 40), (3000, 128, 512), (5000, 640, 128), (70, 8200, 264), (4097, 96, 81),
]


def check_linear(T, N, K, act, bias, residual, eight, out_dtype, preact, x=None, w=None):
    x = rand(1, T, K) if x is None else x
    w = rand(2, N, K) / math.sqrt(K) if w is None else w
    kw = {}
    if eight:
        x, xs = whtmix.quantize_rows(x)
        w, ws = whtmix.quantize_rows(w)
        kw = {"x_scale": xs, "w_scale": ws}
        X, W = x.double() * xs.double()[:, None], w.double() * ws.double()[:, None]
    else:
        x, w = x.to(BF), w.to(BF)
        X, W = x.double(), w.double()
    b = rand(3, N) if bias else None
    r = rand(4, T, N).to(out_dtype) if residual else None
    out, out_ok = guarded((T, N), out_dtype)
    p_out, p_ok = guarded((T, N), BF) if preact else (None, lambda: None)
    got = whtmix.linear(x, w, bias=b, activation=act, residual=r, out_dtype=out_dtype, out=out, preact=p_out, **kw)
    assert (got[0] if preact else got) is out
    out_ok()
    p_ok()
    p = X @ W.T + (b.double() if bias else 0.0)
    size = X.abs() @ W.abs().T
    p_err = K * 2.0 ** -23 * size + 8 * U32 * p.abs()
    y, slope = phi(p, act)
    y_err = 1.2 * p_err + 2.0 ** -17 * y.abs() + 2.0 ** -17 * (p * slope).abs()  # every |slope| <= 1.13
    if residual:
        y = y + r.double()
    unit = U16 if out_dtype == BF else U32
    close(out, y, unit * (1 + U16) * (y.abs() + y_err) + y_err + U32 * y.abs() + 1e-30)
    if preact:
        close(p_out, p, U16 * (1 + U16) * (p.abs() + p_err) + p_err + 1e-30)
    return x, w, p


@pytest.mark.parametrize("T,N,K", LINEAR_SHAPES)
def test_linear_against_float64(T, N, K):
    check_linear(T, N, K, "none", False, False, False, BF, False)
    check_linear(T, N, K, "gelu", True, True, False, BF, True)
    check_linear(T, N, K, "silu", True, False, False, F32, False)
    check_linear(T, N, K, "relu", False, True, False, F32, False)


@pytest.mark.parametrize("T,N,K", LINEAR_SHAPES)
def test_eight_bit_linear_against_float64(T, N, K):
    check_linear(T, N, K, "silu", True, True, True, BF, True)
    check_linear(T, N, K, "none", False, False, True, F32, False)


@pytest.mark.parametrize("T,N,K", [(20011, 304, 136), (20011, 300, 135), (40000, 512, 64), (9000, 520, 384), (9001, 129, 5), (700, 1001, 500)])
def test_products_of_many_tokens_and_short_axes(T, N, K):
    """Several tiles a CTA and few K blocks; residuals of odd rows."""
    for eight in (False, True):
        check_linear(T, N, K, "gelu", True, False, eight, BF, False)
        check_linear(T, N, K, "silu", True, True, eight, BF, True)
        check_linear(T, N, K, "none", False, True, eight, F32, False)


@pytest.mark.parametrize("T,N,K", [(8192, 4096, 1024), (5000, 4100, 2000), (9001, 2048, 1003)])
def test_large_products_against_float64(T, N, K):
    """Long K axes: two CTAs on a tile; the last tiles of rows and columns cut."""
    check_linear(T, N, K, "gelu", True, True, False, BF, True)
    check_linear(T, N, K, "none", True, False, True, F32, False)
    check_linear_backward(T, N, K, "silu")


def test_linear_of_integers_is_exact():
    """Small integers: every product and sum is exact in float32, so that one wrong element shows."""
    g = torch.Generator(device="cuda")
    g.manual_seed(7)
    for T, N, K in [(1, 300, 200), (50, 129, 77), (120, 256, 1024), (300, 777, 333), (2000, 520, 128), (8000, 4096, 1500)]:
        x = torch.randint(-3, 4, (T, K), generator=g, device="cuda").to(BF)
        w = torch.randint(-3, 4, (N, K), generator=g, device="cuda").to(BF)
        b = torch.randint(-9, 10, (N,), generator=g, device="cuda").float()
        r = torch.randint(-9, 10, (T, N), generator=g, device="cuda").float()
        y = whtmix.linear(x, w, bias=b, residual=r, out_dtype=F32)
        assert torch.equal(y.double(), x.double() @ w.double().T + b.double() + r.double())
        ones_x, ones_w = torch.ones(T, device="cuda"), torch.full((N,), 2.0, device="cuda")
        y8 = whtmix.linear(x.to(E4M3), w.to(E4M3), x_scale=ones_x, w_scale=ones_w, out_dtype=F32)
        assert torch.equal(y8.double(), 2 * (x.double() @ w.double().T))
        dy = torch.randint(-3, 4, (T, N), generator=g, device="cuda").to(BF)
        _, dw, db = whtmix.linear_backward(x, w, dy, dw_dtype=F32)
        assert torch.equal(dw.double(), dy.double().T @ x.double()) and torch.equal(db.double(), dy.double().sum(0))


def test_linear_in_place_strided_and_misaligned():
    T, N, K = 200, 256, 192
    w, r = (rand(2, N, K) / 14).to(BF), rand(4, T, N).to(BF)
    wide = rand(1, T, 2 * K + 8).to(BF)
    for start in (0, 8, 3):  # 16-byte aligned rows and rows that are not
        x = wide[:, start:start + K]
        y = whtmix.linear(x, w, residual=r, activation="gelu")
        assert torch.equal(y, whtmix.linear(x.contiguous(), w, residual=r, activation="gelu"))
        buf = r.clone()
        assert torch.equal(whtmix.linear(x, w, residual=buf, activation="gelu", out=buf), y)
    x = wide[:, :K].contiguous()
    y = whtmix.linear(x, w)
    block = torch.zeros(T, 3 * N + 5, dtype=BF, device="cuda")
    whtmix.linear(x, w, out=block[:, N + 1:2 * N + 1])  # a slice of a fused buffer, misaligned
    assert torch.equal(block[:, N + 1:2 * N + 1], y)
    assert bool((block[:, :N + 1] == 0).all()) and bool((block[:, 2 * N + 1:] == 0).all())
    every = torch.zeros(2 * T, N, dtype=BF, device="cuda")
    whtmix.linear(x, w, out=every[::2])
    assert torch.equal(every[::2], y) and bool((every[1::2] == 0).all())
    few = torch.zeros(9, 3 * N + 5, dtype=BF, device="cuda")
    whtmix.linear(x[:9], w, out=few[:, 1:N + 1])
    assert bool((few[:, 0] == 0).all()) and bool((few[:, N + 1:] == 0).all())
    close(few[:, 1:N + 1], y[:9].double(), 2 * U16 * y[:9].double().abs() + 2.0 ** -12)
    # three leading axes
    assert torch.equal(whtmix.linear(x.view(4, 5, 10, K), w), y.view(4, 5, 10, N))


def test_what_lies_between_rows_is_neither_read_nor_written():
    """Rows at a 16-byte pitch that are no whole multiple of 16 bytes: the elements between them are someone else's."""
    for T in (1, 9, 200):
        for K, N in ((300, 129), (67, 1002), (128, 68)):
            kp, np_ = (K + 7) // 8 * 8 + 8, (N + 7) // 8 * 8 + 8
            x, w = torch.full((T, kp), math.nan, device="cuda").to(BF), torch.full((N, kp), math.nan, device="cuda").to(BF)
            x[:, :K], w[:, :K] = rand(1, T, K).to(BF), rand(2, N, K).to(BF)
            y, p, r = (torch.full((T, np_), 7.0, device="cuda").to(BF) for _ in range(3))
            r[:, :N] = rand(3, T, N).to(BF)
            r[:, N:] = math.nan
            whtmix.linear(x[:, :K], w[:, :K], residual=r[:, :N], activation="gelu", preact=p[:, :N], out=y[:, :N])
            want = whtmix.linear(x[:, :K].contiguous(), w[:, :K].contiguous(), residual=r[:, :N].contiguous(), activation="gelu")
            assert torch.equal(y[:, :N], want) and bool((y[:, N:] == 7).all()) and bool((p[:, N:] == 7).all())
            dy = torch.full((T, np_), math.nan, device="cuda").to(BF)
            dy[:, :N] = rand(4, T, N).to(BF)
            dx = torch.full((T, kp), 7.0, device="cuda").to(BF)
            _, dw, db = whtmix.linear_backward(x[:, :K], w[:, :K], dy[:, :N], p[:, :N], "gelu", dx=dx[:, :K])
            assert bool((dx[:, K:] == 7).all())
            got = whtmix.linear_backward(x[:, :K].contiguous(), w[:, :K].contiguous(), dy[:, :N].contiguous(), p[:, :N].contiguous(), "gelu")
            assert torch.equal(dx[:, :K], got[0]) and torch.equal(dw, got[1]) and torch.equal(db, got[2])
            gain = torch.ones(N, device="cuda")
            n, q = torch.full((T, np_), 7.0, device="cuda").to(BF), torch.full((T, np_), 7.0, device="cuda").to(E4M3)
            whtmix.rms_norm(r[:, :N], gain, out=n[:, :N])
            whtmix.rms_norm(r[:, :N], gain, out=q[:, :N], out_dtype=E4M3)
            # (a row's sum of squares is grouped by its distance from a 16-byte boundary: no bits to compare with)
            ref = norm_ref(r[:, :N], None, gain)[1]
            close(n[:, :N], ref, (U16 * (1 + U16) + (N / 32 + 60) * U32 + 2.0 ** -21) * ref.abs() + 1e-37)
            assert bool((n[:, N:] == 7).all()) and bool((q[:, N:].float() == 7).all())


def test_values_that_are_not_finite_stay_where_they_are():
    """An infinity or a NaN in one token or one channel reaches that row or column only, and no neighbour in an epilogue."""
    T, N, K = 150, 200, 96
    w, b = (rand(2, N, K) / 10).to(BF), rand(3, N)
    for t in (150, 20):
        x = rand(1, t, K).to(BF)
        for act in ("none", "relu", "gelu", "silu"):
            clean = whtmix.linear(x, w, bias=b, activation=act)
            bad = x.clone()
            bad[7, 5], bad[9, 1] = math.nan, math.inf
            got = whtmix.linear(bad, w, bias=b, activation=act)
            assert bool(torch.isnan(got[7]).all())
            rest = [i for i in range(t) if i not in (7, 9)]
            assert torch.equal(got[rest], clean[rest])
            bb = b.clone()
            bb[11] = math.nan
            got = whtmix.linear(x, w, bias=bb, activation=act)
            cols = [i for i in range(N) if i != 11]
            assert bool(torch.isnan(got[:, 11]).all()) and torch.equal(got[:, cols], clean[:, cols])
    # far ends of the activations
    z = torch.tensor([-3.0e38, -1.0e30, -1e4, -88.0, -40.0, 0.0, 40.0, 1e4, 1e30, 3e38], device="cuda")
    x1, w1 = torch.zeros(1, 8, device="cuda").to(BF), torch.zeros(len(z), 8, device="cuda").to(BF)
    for act in ("gelu", "silu"):
        y = whtmix.linear(x1, w1, bias=z, activation=act, out_dtype=F32)[0].double()
        close(y, phi(z.double(), act)[0], 2.0 ** -17 * z.double().clamp_min(0) + 1e-15)


def check_linear_backward(T, N, K, act, dw_dtype=BF, seed=0):
    x, w = rand(seed + 1, T, K).to(BF), (rand(seed + 2, N, K) / math.sqrt(K)).to(BF)
    dy = rand(seed + 3, T, N).to(BF)
    p = rand(seed + 4, T, N).to(BF) if act != "none" else None
    dx_o, dx_ok = guarded((T, K), BF)
    dw_o, dw_ok = guarded((N, K), dw_dtype)
    db_o, db_ok = guarded((N,), F32)
    dx, dw, db = whtmix.linear_backward(x, w, dy, p, act, dw_dtype=dw_dtype, dx=dx_o, dw=dw_o, db=db_o)
    dx_ok(), dw_ok(), db_ok()
    dp = dy.double() * (phi(p.double(), act)[1] if act != "none" else 1.0)
    dp_err = 2.0 ** -16 * dy.double().abs()  # the slope in float32
    close(db, dp.sum(0), (T / 16 + 100) * U32 * dp.abs().sum(0) + dp_err.sum(0) * (act != "none") + 1e-30)
    term = U16 * dp.abs() + dp_err if act != "none" else torch.zeros_like(dp)  # dp rounded once
    for got, a, b_, e in ((dx, dp, w.double(), term), (dw, dp.T, x.double(), term.T)):
        ref, size = a @ b_, a.abs() @ b_.abs()
        err = e @ b_.abs() + a.shape[1] * 2.0 ** -23 * size
        unit = U32 if got.dtype == F32 else U16
        close(got, ref, unit * (1 + U16) * (ref.abs() + err) + err + 1e-30)
        # and as a whole: roundings of random sign
        assert float((got.double() - ref).norm()) <= 2 * max(U16 if got.dtype == BF or act != "none" else 2.0 ** -14, 2.0 ** -14) * float(ref.norm() + 1e-30) + 1e-30
    return x, w, dy, p, (dx, dw, db)


@pytest.mark.parametrize("act", ["none", "relu", "gelu", "silu"])
@pytest.mark.parametrize("T,N,K", [(1, 1, 1), (1, 200, 300), (2, 427, 120), (20, 65, 33), (130, 64, 64), (136, 995, 928), (300, 130, 257),
                                   (1000, 256, 128), (2049, 96, 640), (5000, 520, 72), (4000, 33, 1000)])
def test_linear_backward_against_float64(T, N, K, act):
    check_linear_backward(T, N, K, act)
    check_linear_backward(T, N, K, act, dw_dtype=F32)


@pytest.mark.parametrize("act", ["relu", "gelu", "silu"])
@pytest.mark.parametrize("T,N,K", [(9729, 1024, 256), (12000, 200, 130), (20001, 72, 64), (10240, 520, 33)])
def test_linear_backward_of_many_tokens_and_few_channels(T, N, K, act):
    """dp, its sums and dx in one pass."""
    check_linear_backward(T, N, K, act)


def test_linear_backward_of_many_tokens_leaves_out_what_is_not_wanted():
    T, N, K = 10000, 136, 100
    x, w, dy, p, (dx, dw, db) = check_linear_backward(T, N, K, "gelu")
    again = whtmix.linear_backward(x, w, dy, p, "gelu")
    assert torch.equal(dx, again[0]) and torch.equal(dw, again[1]) and torch.equal(db, again[2])
    one = whtmix.linear_backward(x, w, dy, p, "gelu", need_dw=False, need_db=False)
    assert torch.equal(one[0], dx) and one[1] is None and one[2] is None
    two = whtmix.linear_backward(x, w, dy, p, "gelu", need_dw=False)
    assert torch.equal(two[0], dx) and torch.equal(two[2], db)
    bad = dy.clone()
    bad[5000, 3] = math.nan
    got = whtmix.linear_backward(x, w, bad, p, "gelu")
    rest = [i for i in range(T) if i != 5000]
    cols = [i for i in range(N) if i != 3]
    assert bool(torch.isnan(got[0][5000]).all()) and torch.equal(got[0][rest], dx[rest])
    assert bool(torch.isnan(got[1][3]).all()) and torch.equal(got[1][cols], dw[cols])
    assert bool(torch.isnan(got[2][3])) and torch.equal(got[2][cols], db[cols])


def test_linear_backward_repeats_bit_for_bit_and_leaves_out_what_is_not_wanted():
    x, w, dy, p, (dx, dw, db) = check_linear_backward(3000, 200, 128, "gelu")
    again = whtmix.linear_backward(x, w, dy, p, "gelu")
    assert torch.equal(dx, again[0]) and torch.equal(dw, again[1]) and torch.equal(db, again[2])
    one = whtmix.linear_backward(x, w, dy, p, "gelu", need_dw=False, need_db=False)
    assert torch.equal(one[0], dx) and one[1] is None and one[2] is None
    two = whtmix.linear_backward(x, w, dy, p, "gelu", need_dx=False)
    assert two[0] is None and torch.equal(two[1], dw) and torch.equal(two[2], db)
    # strided gradients, misaligned
    wide = torch.zeros(3000, 2 * 200 + 3, dtype=BF, device="cuda")
    wide[:, 1:201] = dy
    got = whtmix.linear_backward(x, w, wide[:, 1:201], p, "gelu")
    assert torch.equal(got[0], dx) and torch.equal(got[1], dw)


def test_linear_gradients_by_differences():
    """Against central differences of the float64 definition, through autograd; values that bf16 holds, small sizes."""
    T, N, K = 4, 16, 24
    x, w, b, r, dy = rand(1, T, K).to(BF), (rand(2, N, K) / 5).to(BF), rand(3, N), rand(4, T, N).to(BF), rand(5, T, N).to(BF)

    def loss(x_, w_, b_, act):
        return float(((phi(x_ @ w_.T + b_, act)[0] + r.double()) * dy.double()).sum())

    for act in ("none", "gelu", "silu"):
        leaves = [t.clone().requires_grad_(True) for t in (x, w, b, r)]
        y = whtmix.LinearFunction.apply(*leaves, act)
        (y.float() * dy.float()).sum().backward()
        assert torch.equal(leaves[3].grad, dy)
        step = 1e-5
        base = [x.double(), w.double(), b.double()]
        for which in range(3):
            grad = leaves[which].grad.double()
            # p is stored in bf16 (2^-9 |p| times a slope of at most 1.2), dp rounded, the result rounded
            tol = 6 * U16 * float(grad.abs().max()) + 1e-4
            for i in range(0, base[which].numel(), 7):
                d = torch.zeros_like(base[which]).view(-1)
                d[i] = step
                d = d.view(base[which].shape)
                up, down = [v.clone() for v in base], [v.clone() for v in base]
                up[which] += d
                down[which] -= d
                diff = (loss(*up, act) - loss(*down, act)) / (2 * step)
                assert abs(diff - float(grad.reshape(-1)[i])) <= tol


def test_nothing_to_do():
    w, gain = (rand(2, 64, 32) / 5).to(BF), torch.ones(32, device="cuda")
    x = torch.empty(0, 32, dtype=BF, device="cuda")
    y, h = whtmix.rms_norm(x, gain, residual=x)
    assert y.shape == (0, 32) and h.shape == (0, 32)
    assert whtmix.linear(x, w).shape == (0, 64)
    dx, dw = whtmix.rms_norm_backward(x, gain, x)
    assert dx.shape == (0, 32) and bool((dw == 0).all())
    dx, dw, db = whtmix.linear_backward(x, w, torch.empty(0, 64, dtype=BF, device="cuda"))
    assert dx.shape == (0, 32) and bool((dw == 0).all()) and bool((db == 0).all())


def test_on_another_stream_and_in_a_graph():
    T, N, K = 300, 256, 200
    gain, w, b = torch.ones(K, device="cuda"), (rand(2, N, K) / 14).to(BF), rand(3, N)
    x, r, dy = rand(1, T, K).to(BF), rand(4, T, K).to(BF), rand(5, T, N).to(BF)

    def layer(stream=None):
        y, h = whtmix.rms_norm(x, gain, residual=r, stream=stream)
        z, p = whtmix.linear(y, w, bias=b, activation="gelu", preact=True, stream=stream)
        dx, dw, db = whtmix.linear_backward(y, w, dy, p, "gelu", stream=stream)
        dn, dg = whtmix.rms_norm_backward(h, gain, dx, stream=stream)
        return z, dw, db, dn, dg

    want = layer()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got = layer()
    whtmix.sync(s)
    assert all(torch.equal(a, b_) for a, b_ in zip(got, want))
    got = layer(stream=s)
    whtmix.sync(s)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b_) for a, b_ in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        got = layer()
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b_) for a, b_ in zip(got, want))


@pytest.mark.parametrize("lead", [(1,), (5, 7), (130,)])
def test_calls_with_and_without_given_results_agree(lead):
    """The compiled path of plain calls and the step-by-step one (results given) launch the same work."""
    K, N = 96, 80
    x, r = rand(1, *lead, K).to(BF), rand(2, *lead, K).to(BF)
    gain = 1.0 + 0.1 * rand(3, K)
    new = lambda *shape, dtype=BF: torch.empty(*shape, dtype=dtype, device="cuda")
    y, h = whtmix.rms_norm(x, gain, residual=r)
    y2, h2 = whtmix.rms_norm(x, gain, residual=r, out=new(*lead, K), h=new(*lead, K))
    assert torch.equal(y, y2) and torch.equal(h, h2)
    assert torch.equal(whtmix.rms_norm(h, gain), whtmix.rms_norm(h, gain, out=new(*lead, K)))
    q, s, h3 = whtmix.rms_norm(x, gain, residual=r, out_dtype=E4M3)
    q2, s2, _ = whtmix.rms_norm(x, gain, residual=r, out_dtype=E4M3, scale=new(*lead, dtype=F32))
    assert torch.equal(q.float(), q2.float()) and torch.equal(s, s2) and torch.equal(h, h3)
    dx, dw = whtmix.rms_norm_backward(h, gain, x, dh=r)
    dx2, dw2 = whtmix.rms_norm_backward(h, gain, x, dh=r, dx=new(*lead, K))
    assert torch.equal(dx, dx2) and torch.equal(dw, dw2)
    w, b, res = rand(4, N, K).to(BF), rand(5, N), rand(6, *lead, N).to(BF)
    z, p = whtmix.linear(x, w, b, "gelu", residual=res, preact=True)
    z2, p2 = whtmix.linear(x, w, b, "gelu", residual=res, preact=True, out=new(*lead, N))
    assert torch.equal(z, z2) and torch.equal(p, p2) and z.shape == (*lead, N)
    assert torch.equal(whtmix.linear(x, w, b, "gelu", residual=res, preact=False), z)
    wq, ws = whtmix.quantize_rows(w)
    eight = whtmix.linear(q, wq, b, "silu", x_scale=s, w_scale=ws, out_dtype=F32)
    again = whtmix.linear(q, wq, b, "silu", x_scale=s, w_scale=ws, out_dtype=F32, out=new(*lead, N, dtype=F32))
    assert eight.dtype == F32 and torch.equal(eight, again)
    for need in ((True, True, True), (1, 0, 1), (False, True, False)):
        got = whtmix.linear_backward(x, w, res, p, "gelu", *need, dw_dtype=F32)
        all_given = whtmix.linear_backward(x, w, res, p, "gelu", dw_dtype=F32, dx=new(*lead, K))
        for g, a, wanted in zip(got, all_given, need):
            assert (g is None) if not wanted else torch.equal(g, a)


def test_a_streams_first_call_may_be_the_smallest():
    """A stream's first workspace for a call that needs a few bytes."""
    x, w, dy = rand(1, 1, 1), torch.ones(1, device="cuda"), rand(2, 1, 1)
    whtmix.release_workspaces()
    check_norm_backward(x, w, dy, None)
    for T, N, K in ((1, 1, 1), (3, 2, 5)):
        a, b, g = rand(1, T, K).to(BF), rand(2, N, K).to(BF), rand(3, T, N).to(BF)
        whtmix.release_workspaces()
        y = whtmix.linear(a, b)
        whtmix.release_workspaces()
        dx, dw, db = whtmix.linear_backward(a, b, g, need_db=True)
        whtmix.sync()
        A, B, G = a.double(), b.double(), g.double()
        for got, left, right in ((y, A, B.T), (dx, G, B), (dw, G.T, A), (db, torch.ones(1, T, device="cuda").double(), G)):
            ref = (left @ right).reshape(got.shape)
            close(got, ref, U16 * 1.01 * ref.abs() + 2.0 ** -18 * (left.abs() @ right.abs()).reshape(got.shape))


def test_offsets_beyond_32_bits():
    """Rows at more than 2^31 and 2^32 elements: the first, one past each and the last are right."""
    T, D = (1 << 32) // 4096 + 70, 4096
    x = torch.zeros(T, D, dtype=BF, device="cuda")  # 8.6 GB
    rows = [0, (1 << 31) // D + 1, (1 << 32) // D + 3, T - 1]
    for i, t in enumerate(rows):
        x[t] = rand(i, D).to(BF)
    gain, w = torch.ones(D, device="cuda"), (rand(2, 64, D) / 64).to(BF)
    picked = x[rows]
    y = whtmix.linear(x, w)
    close(y[rows], picked.double() @ w.double().T, U16 * 1.01 * (picked.double() @ w.double().T).abs() + D * 2.0 ** -23 * (picked.double().abs() @ w.double().abs().T))
    assert float(y.float().abs().sum()) == float(y[rows].float().abs().sum())
    dy = torch.zeros(T, 64, dtype=BF, device="cuda")
    dy[rows] = rand(9, 4, 64).to(BF)
    _, dw, _ = whtmix.linear_backward(x, w, dy, need_dx=False, dw_dtype=F32)
    ref = dy[rows].double().T @ picked.double()
    close(dw, ref, 2.0 ** -18 * (dy[rows].double().abs().T @ picked.double().abs()) + 1e-30)
    n = whtmix.rms_norm(x, gain, out=x)
    close(n[rows], norm_ref(picked, None, gain)[1], 1.02 * U16 * norm_ref(picked, None, gain)[1].abs())
