"""Layer norm at its edges on a GPU, against plain float64 implementations: finite rows of any size of values, and 8-bit rows without
residual and shift.

Tolerances as test_train_ops_gpu.py derives them: they are relative to a row's values (c, the variance, rstd), so that they hold for a row
times a power of two as they do for the row.  What leaves float32's normal range on the way out is off by 2^-149 at most, below the
1e-37 that `rounded` allows."""
import math

import pytest
import torch

from paper_2607_25234_gb300 import whtmix
from test_train_ops_gpu import BF, E4M3, EPS, F32, U16, U32, Norm, close, device, e4m3_step, guarded, norm_inputs, rand, rounded  # noqa: F401

pytestmark = pytest.mark.gpu

# row i is of size SIZES[i % 9]: squares beyond float32 on either side, sums beyond it, and rows in range among them
SIZES = [1.0, 1e18, 1e25, 3e37, 1e-25, 1.0, 1e-36, 1e19, 1e-15]
# (rows, channels): every row kernel, aligned and not, few and many rows, rows beyond the registers, tiles, tiles of wide rows
SHAPES = [(9, 16), (40, 64), (18, 128), (400, 128), (27, 256), (200, 256), (200, 512), (27, 1000), (200, 1024), (160, 1536), (20, 2048), (160, 2560),
          (18, 4096), (160, 4096), (18, 6144), (18, 8192), (9, 16384), (18, 16392), (18, 7), (40, 77), (200, 301), (27, 1001), (701, 1501), (18, 2999),
          (18, 5001), (9, 8191), (9, 12001), (9, 20001), (10001, 9), (9737, 50), (20011, 77), (4900, 177), (5000, 301), (2440, 499), (2500, 601),
          (2433, 765), (2500, 1001), (2441, 1277), (2500, 1501), (2440, 2047)]


def sized(x):
    """x with its rows at SIZES."""
    by = torch.tensor(SIZES, dtype=torch.float64, device="cuda")[torch.arange(x.shape[0], device="cuda") % len(SIZES)]
    return (x.double() * by[:, None]).to(x.dtype)


@pytest.mark.parametrize("eps", [EPS, 0.0])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T,D", SHAPES)
def test_finite_rows_have_their_norm_whatever_their_size(T, D, dtype, eps):
    x, res, w, b = norm_inputs(T, D, dtype)
    x, res = sized(x), sized(res)
    for residual, shift in ((None, b), (res, None)):
        got = whtmix.layer_norm(x, w, shift, residual=residual, eps=eps)
        h = x.double() if residual is None else x.double() + residual.double()
        y, err = Norm(h, eps).y(w, shift)
        close(got if residual is None else got[0], y, rounded(y, err, dtype))
        if residual is not None:
            close(got[1], h, rounded(h, U32 * h.abs(), dtype))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T,D", SHAPES)
def test_finite_rows_to_eight_bits_whatever_their_size(T, D, dtype):
    x, _, w, _ = norm_inputs(T, D, dtype)
    for eps, rows in ((0.0, sized(x)), (EPS, x)):  # neither residual nor shifts: one matrix a stage where rows come as tiles
        q, scale = whtmix.layer_norm(rows, w, eps=eps, out_dtype=E4M3)
        y, err = Norm(rows, eps).y(w, None)
        s = y.abs().amax(-1, keepdim=True) / 448.0
        s_err = err.amax(-1, keepdim=True) / 448.0 + 2 * U32 * s
        close(scale[:, None], s, s_err)
        v = y / s
        v_err = err / s + v.abs() * s_err / s + 4 * U32 * v.abs()
        close(q.float(), v, (e4m3_step(v) / 2 + v_err) * (1 + 2.0 ** -12))


@pytest.mark.parametrize("eps", [EPS, 0.0])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T,D", SHAPES)
def test_finite_rows_have_their_gradients_whatever_their_size(T, D, dtype, eps):
    h, _, w, _ = norm_inputs(T, D, dtype)
    h, dy = sized(h), rand(5, T, D).to(dtype)
    ref = Norm(h, eps)
    mean = lambda v: v.mean(-1, keepdim=True)
    G = dy.double()
    a = G * w.double()
    n, n_err, an = ref.n, ref.n_err, a * ref.n
    want = ref.rstd * (a - mean(a) - n * mean(an))
    spread = ref.rstd * (a.abs() + mean(a.abs()) + n.abs() * mean(an.abs()))
    err = ref.rstd * (n_err * mean(an.abs()) + n.abs() * mean(a.abs() * n_err)) + (3 * ref.rel + ref.sum_err + 12 * U32) * spread
    # (gradients beyond the type are infinite, and those next to its largest value may be)
    top = 3.0e38
    seen = (want.abs() + err) * (1 + 2 * U16) < top
    rows = (T / 32 + D / 32 + 200) * U32
    for dh in (None, rand(6, T, D).to(dtype)):
        total = want if dh is None else want + dh.double()
        total_err = err if dh is None else err + U32 * (dh.double().abs() + spread)
        dx, dw, db = whtmix.layer_norm_backward(h, w, dy, dh=dh, eps=eps)
        close(torch.where(seen, dx.double(), 0.0), torch.where(seen, total, 0.0), rounded(total, total_err, dtype))
        close(dw, (G * n).sum(0), rows * (G * n).abs().sum(0) + (G.abs() * n_err).sum(0) + 4 * U32 * (G * n).abs().sum(0) + 1e-37)
        close(db, G.sum(0), rows * G.abs().sum(0) + 1e-37)
        for over in ("dy", "dh") if dh is not None else ("dy",):  # dx in another's place
            p, q = dy.clone(), None if dh is None else dh.clone()
            again = whtmix.layer_norm_backward(h, w, p, dh=q, dx=p if over == "dy" else q, eps=eps)
            assert all(torch.equal(u, v) for u, v in zip(again, (dx, dw, db)))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("D", [32, 64, 128, 256, 1024, 77, 1001])
@pytest.mark.parametrize("T", [20, 20000])
def test_rows_of_any_size_in_place(T, D, dtype):
    if T * D > 1 << 22 and D > 128:
        T = 3000
    x, r, w, b = norm_inputs(T, D, dtype)
    x, r = sized(x), sized(r)
    want_y, want_h = whtmix.layer_norm(x, w, b, residual=r)
    alone = whtmix.layer_norm(x, w, b)
    a = x.clone()
    assert torch.equal(whtmix.layer_norm(a, w, b, out=a), alone)
    for target in ("x", "r"):
        p, q = x.clone(), r.clone()
        y, h = whtmix.layer_norm(p, w, b, residual=q, h=p if target == "x" else q)
        assert torch.equal(y, want_y) and torch.equal(h, want_h)
        p, q = x.clone(), r.clone()
        y, h = whtmix.layer_norm(p, w, b, residual=q, out=p if target == "x" else q)
        assert torch.equal(y, want_y) and torch.equal(h, want_h)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T,D", [(6, 64), (6, 256), (6, 1000), (6, 1024), (6, 4096), (6, 8192), (6, 20001), (20011, 77), (2500, 1001)])
def test_large_equal_values_and_rows_that_are_not_finite(T, D, dtype):
    w, b, dy = 1.0 + 0.1 * rand(3, D), 0.1 * rand(4, D), rand(5, T, D).to(dtype)
    x = rand(1, T, D).to(dtype)
    y0, (dx0, _, _) = whtmix.layer_norm(x, w, b), whtmix.layer_norm_backward(x, w, dy)
    x[0] = 3.0e38  # their sum is infinite
    x[1] = 2.0 ** 40
    x[2, D // 3] = math.inf
    x[3] = 1e25
    x[3, D // 2] = math.nan
    x[4] = -1e33
    y, (dx, dw, db) = whtmix.layer_norm(x, w, b), whtmix.layer_norm_backward(x, w, dy)
    for i in (0, 1, 4):
        ref, err = Norm(x[i:i + 1]).y(w, b)
        # c is the rounding of the mean, y at most as the largest normalised value
        close(y[i:i + 1], ref, rounded(ref, torch.minimum(err, w.double().abs() * math.sqrt(D) * 1.001), dtype))
        assert bool(torch.isfinite(dx[i]).all())
    if D & (D - 1) == 0:  # the mean is exact where every partial sum is: up to 2^16 equal values of 8 bits, any of 2^40 (three of 24 bits take 26)
        exact = [0, 1, 4] if dtype == BF else [1]
        assert torch.equal(y[exact], b.to(dtype).expand(len(exact), D))
    for i in (2, 3):
        assert bool(torch.isnan(y[i]).all()) and bool(torch.isnan(dx[i]).all())
    assert bool(torch.isnan(dw).all()) and bool(torch.isfinite(db).all())
    assert torch.equal(y[5:], y0[5:]) and torch.equal(dx[5:], dx0[5:])  # the neighbours
    q, scale = whtmix.layer_norm(x, w, b, out_dtype=E4M3)
    assert bool(torch.isfinite(scale[[0, 1, 4, 5]]).all()) and bool(torch.isnan(scale[2:4]).all())
    assert bool(torch.isnan(q[2:4].float()).all()) and bool(torch.isfinite(q[[0, 1, 4, 5]].float()).all())


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T,D", [(5, 16), (300, 16), (5, 48), (5, 200), (5, 1000), (300, 1000), (5, 77), (5, 1001), (5, 4100), (20011, 77)])
def test_large_equal_values_with_a_small_eps_to_eight_bits(T, D, dtype):
    """mean rstd leaves float32 here; places that are not the row's must not see it.  2^100 is its own mean where D is a power of two; else
    the mean's rounding is the row's c, whose norm is at most sqrt(D)."""
    w, b = 1.0 + 0.1 * rand(3, D), 0.1 * rand(4, D)
    x = torch.full((T, D), 2.0 ** 100, device="cuda").to(dtype)
    q, scale = whtmix.layer_norm(x, w, b, eps=1e-30, out_dtype=E4M3)
    y = whtmix.layer_norm(x, w, b, eps=1e-30)
    top = float((w.abs() * math.sqrt(D) + b.abs()).max()) * 1.001
    assert bool(torch.isfinite(scale).all()) and float(scale.max()) <= top / 448.0 and bool(torch.isfinite(q.float()).all())
    assert bool(torch.isfinite(y).all()) and float(y.float().abs().max()) <= top * (1 + U16)
    if D & (D - 1) == 0:
        assert torch.equal(scale, b.abs().max().expand(T) * (1.0 / 448.0)) and torch.equal(y, b.to(dtype).expand(T, D))
