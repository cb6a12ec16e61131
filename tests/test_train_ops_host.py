"""Refusals of layer norm, the gated feed-forward half and clipping by a common norm: the C entry points and the binding (CPU)."""
import ctypes
import re

import pytest
import torch

from paper_2607_25234_gb300 import build as libbuild
from paper_2607_25234_gb300 import whtmix
from test_capi_host import FAKE, passes_every_check
from test_layer_host import waits_before_it_ends
from test_ordering_host import functions, read

INVALID, SHAPE, DTYPE, ALIGN, ALIAS = 1, 2, 3, 4, 5


@pytest.fixture(scope="module")
def lib():
    libbuild.build()
    return whtmix.library()


def norm(lib, x=FAKE, r=2 * FAKE, w=3 * FAKE, b=8 * FAKE, h=4 * FAKE, y=5 * FAKE, s=None, T=4, D=8, xs=8, rs=8, hs=8, ys=8, eps=1e-5, dt=1, odt=1):
    return lib.whtmix_layer_norm(x, r, w, b, h, y, s, T, D, xs, rs, hs, ys, eps, dt, odt, None)


def norm_bwd(lib, h=FAKE, w=2 * FAKE, dy=3 * FAKE, dh=4 * FAKE, dx=5 * FAKE, dw=6 * FAKE, db=7 * FAKE, T=4, D=8, hs=8, ys=8, gs=8, xs=8, eps=1e-5,
             dt=1):
    return lib.whtmix_layer_norm_backward(h, w, dy, dh, dx, dw, db, T, D, hs, ys, gs, xs, eps, dt, None)


def gated(lib, x=FAKE, w=2 * FAKE, sx=None, sw=None, b=3 * FAKE, p=5 * FAKE, y=6 * FAKE, T=4, N=8, K=16, xs=16, ws=16, ps=16, ys=8, act=3, dt=1, odt=1):
    return lib.whtmix_gated_linear(x, w, sx, sw, b, p, y, T, N, K, xs, ws, ps, ys, act, dt, odt, None)


def gated_bwd(lib, x=FAKE, w=2 * FAKE, dy=3 * FAKE, p=4 * FAKE, dx=5 * FAKE, dw=6 * FAKE, db=7 * FAKE, T=4, N=8, K=16, xs=16, ws=16, ys=8, ps=16,
              dxs=16, act=3, wdt=1):
    return lib.whtmix_gated_linear_backward(x, w, dy, p, dx, dw, db, T, N, K, xs, ws, ys, ps, dxs, act, wdt, None)


def tensors(*entries):
    """whtmix_tensor_t of (in, out, n, dtype)."""
    return (whtmix._Tensor * max(len(entries), 1))(*[whtmix._Tensor(*e) for e in entries])


def clip(lib, *entries, count=None, max_norm=1.0, norm=9 * FAKE):
    return lib.whtmix_clip_by_global_norm(tensors(*entries), len(entries) if count is None else count, max_norm, norm, None)


def test_layer_norm_rejects_bad_arguments(lib):
    for call in (norm, norm_bwd):
        assert call(lib, w=None) == INVALID
        assert call(lib, T=-1) == INVALID
        assert call(lib, D=0) == INVALID
        assert call(lib, eps=-1.0) == INVALID
        assert call(lib, eps=float("nan")) == INVALID
        assert call(lib, D=(1 << 24) + 1) == SHAPE
        assert call(lib, T=(1 << 31) - 255) == SHAPE
        assert call(lib, T=1 << 30, D=1 << 11) == SHAPE
        assert call(lib, xs=7) == INVALID
        assert call(lib, xs=1 << 41) == SHAPE
        assert call(lib, dt=2) == DTYPE
        assert call(lib, dt=3) == DTYPE
        passes_every_check(lambda c=call: c(lib))
        passes_every_check(lambda c=call: c(lib, T=1, xs=0))  # one row has no stride
        passes_every_check(lambda c=call: c(lib, **({"b": None} if c is norm else {"db": None, "dh": None})))
    assert norm(lib, x=None) == INVALID and norm(lib, y=None) == INVALID
    assert norm(lib, odt=0) == DTYPE
    assert norm(lib, odt=3) == INVALID  # 8 bits without scales
    assert norm(lib, x=FAKE + 1) == ALIGN and norm(lib, b=8 * FAKE + 2) == ALIGN and norm(lib, odt=3, s=7 * FAKE + 2) == ALIGN
    passes_every_check(lambda: norm(lib, odt=3, s=7 * FAKE, y=5 * FAKE + 1))
    passes_every_check(lambda: norm(lib, r=None, h=None))
    assert norm(lib, x=None, r=None, w=None, b=None, h=None, y=None, T=0) == 0
    assert norm_bwd(lib, dy=None) == INVALID and norm_bwd(lib, dx=None) == INVALID
    assert norm_bwd(lib, dw=None) == INVALID and norm_bwd(lib, dw=None, T=0) == INVALID
    assert norm_bwd(lib, db=7 * FAKE + 2) == ALIGN
    row = 8 * 2  # bytes of a row of 8 bf16
    assert norm(lib, y=FAKE + row) == ALIAS and norm(lib, h=4 * FAKE, y=4 * FAKE) == ALIAS
    assert norm(lib, y=3 * FAKE) == ALIAS and norm(lib, y=8 * FAKE) == ALIAS  # over the gains, over the shifts
    assert norm(lib, y=FAKE, ys=16) == ALIAS
    assert norm(lib, odt=3, s=7 * FAKE, y=FAKE) == ALIAS
    passes_every_check(lambda: norm(lib, y=FAKE))
    passes_every_check(lambda: norm(lib, h=2 * FAKE))
    assert norm_bwd(lib, dx=FAKE) == ALIAS and norm_bwd(lib, dw=FAKE + 16) == ALIAS and norm_bwd(lib, db=6 * FAKE + 4) == ALIAS
    passes_every_check(lambda: norm_bwd(lib, dx=3 * FAKE))
    passes_every_check(lambda: norm_bwd(lib, dx=4 * FAKE))


def test_gated_rejects_bad_arguments(lib):
    for name in ("x", "w", "y"):
        assert gated(lib, **{name: None}) == INVALID
    for name in ("dy", "p", "x", "w"):
        assert gated_bwd(lib, **{name: None}) == INVALID
    for call in (gated, gated_bwd):
        assert call(lib, K=0) == INVALID and call(lib, N=0) == INVALID and call(lib, N=-1) == INVALID and call(lib, N=-(1 << 63)) == INVALID
        assert call(lib, T=-1) == INVALID and call(lib, act=4) == INVALID and call(lib, act=-1) == INVALID
        assert call(lib, N=(1 << 23) + 1) == SHAPE and call(lib, N=1 << 22, K=1 << 22) == SHAPE and call(lib, T=(1 << 31) - 255) == SHAPE
        assert call(lib, xs=15) == INVALID and call(lib, ys=7) == INVALID and call(lib, ps=15) == INVALID
        assert call(lib, p=5 * FAKE + 1) == ALIGN
        passes_every_check(lambda c=call: c(lib))
        passes_every_check(lambda c=call: c(lib, act=0))
    assert gated(lib, sx=8 * FAKE) == INVALID  # scales belong to 8-bit operands
    assert gated(lib, dt=3) == INVALID         # which need them
    passes_every_check(lambda: gated(lib, dt=3, sx=8 * FAKE, sw=9 * FAKE))
    assert gated(lib, dt=0) == DTYPE and gated(lib, odt=2) == DTYPE
    assert gated(lib, odt=0) == DTYPE          # the pre-activations go with a bf16 output
    passes_every_check(lambda: gated(lib, odt=0, p=None, y=6 * FAKE))
    passes_every_check(lambda: gated(lib, b=None, p=None))
    assert gated(lib, b=3 * FAKE + 2) == ALIGN
    assert gated(lib, x=None, w=None, y=None, T=0) == 0
    assert gated(lib, y=FAKE) == ALIAS and gated(lib, y=2 * FAKE + 16) == ALIAS and gated(lib, p=6 * FAKE) == ALIAS
    assert gated(lib, y=5 * FAKE + 16) == ALIAS  # inside the pre-activations
    assert gated_bwd(lib, dx=None, dw=None, db=None) == INVALID
    assert gated_bwd(lib, dx=None, dw=None, db=None, T=0) == 0
    assert gated_bwd(lib, wdt=3) == DTYPE and gated_bwd(lib, dw=6 * FAKE + 1) == ALIGN
    passes_every_check(lambda: gated_bwd(lib, x=None, dw=None))
    passes_every_check(lambda: gated_bwd(lib, w=None, dx=None))
    assert gated_bwd(lib, dx=FAKE) == ALIAS and gated_bwd(lib, dx=3 * FAKE) == ALIAS and gated_bwd(lib, dx=4 * FAKE) == ALIAS
    assert gated_bwd(lib, db=6 * FAKE + 4) == ALIAS


def test_clipping_rejects_bad_arguments(lib):
    a = (FAKE, 3 * FAKE, 1000, 0)
    assert lib.whtmix_global_norm(None, 1, 9 * FAKE, None) == INVALID
    assert lib.whtmix_global_norm(tensors(a), 1, None, None) == INVALID
    assert lib.whtmix_global_norm(tensors(a), -1, 9 * FAKE, None) == INVALID
    passes_every_check(lambda: lib.whtmix_global_norm(tensors((FAKE, None, 1000, 0), (FAKE, None, 1000, 0)), 2, 9 * FAKE, None))  # twice the same
    assert lib.whtmix_global_norm(tensors(a), 1, FAKE + 4, None) == ALIAS
    passes_every_check(lambda: clip(lib, a))
    passes_every_check(lambda: clip(lib, a, norm=None))
    passes_every_check(lambda: clip(lib, (FAKE, FAKE, 1000, 0)))  # in place
    passes_every_check(lambda: clip(lib, a, max_norm=float("inf")))
    assert clip(lib, a, max_norm=-1.0) == INVALID and clip(lib, a, max_norm=float("nan")) == INVALID
    assert clip(lib, a, count=(1 << 20) + 1) == SHAPE
    assert clip(lib, (FAKE, 3 * FAKE, -1, 0)) == INVALID
    assert clip(lib, (FAKE, 3 * FAKE, (1 << 40) + 1, 0)) == SHAPE
    assert clip(lib, (None, 3 * FAKE, 5, 0)) == INVALID and clip(lib, (FAKE, None, 5, 0)) == INVALID
    assert clip(lib, (FAKE, 3 * FAKE, 5, 2)) == DTYPE and clip(lib, (FAKE, 3 * FAKE, 0, 3)) == DTYPE
    assert clip(lib, (FAKE + 2, 3 * FAKE, 5, 0)) == ALIGN and clip(lib, (FAKE, 3 * FAKE + 1, 5, 1)) == ALIGN and clip(lib, a, norm=9 * FAKE + 2) == ALIGN
    passes_every_check(lambda: clip(lib, (FAKE + 2, 3 * FAKE + 6, 5, 1)))
    assert clip(lib, (FAKE, FAKE + 4, 1000, 0)) == ALIAS                                     # over its own input, shifted
    assert clip(lib, (FAKE, FAKE, 1000, 0), (FAKE, FAKE, 1000, 0)) == ALIAS                   # the same tensor twice, in place
    assert clip(lib, a, (FAKE, 5 * FAKE, 1000, 0)) != ALIAS                                   # twice read, written apart
    assert clip(lib, a, (5 * FAKE, 3 * FAKE + 2000, 7, 1)) == ALIAS                           # two outputs
    assert clip(lib, a, (3 * FAKE + 3996, 5 * FAKE, 7, 1)) == ALIAS                           # an output over another's input
    assert clip(lib, a, (3 * FAKE + 4000, 5 * FAKE, 7, 1)) != ALIAS                           # just behind it
    assert clip(lib, a, norm=3 * FAKE + 8) == ALIAS and clip(lib, a, norm=FAKE) == ALIAS
    assert clip(lib, (None, None, 0, 0), norm=None) == 0 and clip(lib, count=0, norm=None) == 0


def test_binding_checks_what_a_pointer_cannot_carry():
    bf, f32, e4 = torch.bfloat16, torch.float32, torch.float8_e4m3fn
    x, w, gain = torch.zeros(4, 16, dtype=bf), torch.zeros(8, 16, dtype=bf), torch.ones(16)
    p, dy = torch.zeros(4, 8, dtype=bf), torch.zeros(4, 4, dtype=bf)
    for call in (lambda: whtmix.layer_norm(x, gain), lambda: whtmix.layer_norm_backward(x, gain, x), lambda: whtmix.gated_linear(x, w),
                 lambda: whtmix.gated_linear_backward(x, w, dy, p), lambda: whtmix.global_norm([x]), lambda: whtmix.clip_by_global_norm([x], 1.0)):
        with pytest.raises(ValueError, match="CUDA"):
            call()
    with pytest.raises(TypeError):
        whtmix.layer_norm(x.to(torch.float16), gain)
    with pytest.raises(TypeError):
        whtmix.layer_norm(x, gain, out_dtype=f32)
    with pytest.raises(TypeError):
        whtmix.layer_norm_backward(x.to(torch.float16), gain, x)
    with pytest.raises(TypeError):
        whtmix.gated_linear(x.float(), w.float())
    with pytest.raises(TypeError):
        whtmix.gated_linear(x, w, out_dtype=torch.float16)
    with pytest.raises(TypeError):
        whtmix.gated_linear_backward(x, w, dy, p, dw_dtype=torch.float16)
    with pytest.raises(ValueError, match="activation"):
        whtmix.gated_linear(x, w, activation="tanh")
    with pytest.raises(ValueError, match="activation"):
        whtmix.gated_linear_backward(x, w, dy, p, activation="elu")
    with pytest.raises(ValueError, match="empty"):
        whtmix.global_norm([])
    with pytest.raises(ValueError, match="empty"):
        whtmix.clip_by_global_norm([], 1.0)
    with pytest.raises(TypeError, match="list of tensors"):
        whtmix.global_norm([gain, 1.0])
    with pytest.raises(ValueError, match="for each"):
        whtmix.clip_by_global_norm([FakeCuda()], 1.0, out=[gain, gain])
    with pytest.raises(ValueError, match="negative"):
        whtmix.clip_by_global_norm([FakeCuda()], -1.0)
    with pytest.raises(ValueError, match="negative"):
        whtmix.clip_by_global_norm([FakeCuda()], float("nan"))
    for bad in (torch.zeros(7, 16, dtype=bf), torch.zeros(8, 15, dtype=bf), torch.zeros(0, 16, dtype=bf), torch.zeros(16, dtype=bf), w.to(e4)):
        with pytest.raises(ValueError, match="w must be"):
            whtmix._halves(bad, bf, 16)
    assert whtmix._halves(w, bf, 16) == (4, 16)


class FakeCuda(torch.Tensor):
    """A tensor that says it is on a GPU, for checks that come before anything else."""
    is_cuda = True


def test_dense_tensors_are_those_of_one_piece():
    t = torch.zeros(4, 5, 6)
    for good in (t, t.permute(2, 0, 1), t.reshape(120), t[:1], t[1:3], torch.zeros(()), torch.zeros(1, 7, 1).expand(1, 7, 1), t[:, :, :0][:0]):
        assert good.numel() == 0 or whtmix._dense(good)
    for bad in (t[:, 1:3], t[..., ::2], t[:, :, :1], torch.zeros(1, 5).expand(3, 5), t[::2]):
        assert not whtmix._dense(bad)


def test_the_table_entry_is_the_headers():
    """whtmix_tensor_t as the binding lays it out: two pointers, a 64-bit count, an int."""
    assert ctypes.sizeof(whtmix._Tensor) == 32
    assert [getattr(whtmix._Tensor, f).offset for f in ("in_", "out", "n", "dtype")] == [0, 8, 16, 24]
    text = open(libbuild.INCLUDE + "/whtmix.h").read()
    body = re.search(r"typedef struct \{([^}]*)\} whtmix_tensor_t;", text).group(1)
    assert re.findall(r"(\w+);", body) == ["in", "out", "n", "dtype"]


def test_copies_and_products_in_flight_are_waited_for_whichever_wait_gave_up():
    text = dict(functions(read("whtmix_gemm_gated.cuh")))["k_gated"]
    assert waits_before_it_ends(text)


def test_the_fused_backwards_copies_and_products_are_waited_for():
    """Its three rings: the inputs' and W's copies by their own barriers, the products by their accumulators', dp's way out by its group."""
    text = dict(functions(read("whtmix_gemm_gated_dp.cu")))["k_dx_gated"]
    for name, first, last in (("full", "if (warp == 0) {\n    if (lane", "else if (warp == 2)"), ("wfull", "else if (warp == 2)", "else if (warp == 1)"),
                              ("dfull", "else if (warp == 1)", "else if (warp == 3)")):
        part = text[text.index(first):text.index(last)]
        tail = part[part.rindex("for (uint32_t j ="):]
        assert re.search(r"j < (it|i); \+\+j\)\s*if \(!tma::wait\(&bars\.%s\[" % name, tail), name
        assert tail.count("bad") == 1  # (waited for whichever wait gave up)
    part = text[text.index("else if (warp == 3)"):text.index("else if (warp >= 8)")]
    assert part.rindex("tma::wait_done();") > part.rindex("tma::store_2d(")
    assert text.index("bars.dempty[d]", text.index("else if (warp >= 4)")) > 0 and text.rindex("tmem_dealloc") > text.rindex("__syncthreads")


def test_tables_of_tensors_fit_a_kernels_parameters():
    """An entry is 32 bytes (two pointers, a size, a chunk); 32,764 bytes is the most a launch can pass."""
    text = read("whtmix_clip.cu")
    few, many = (int(v) for v in re.search(r"FEW = (\d+), MANY = (\d+)", text).groups())
    assert few < many and 32 * many + 8 + 64 <= 32764
