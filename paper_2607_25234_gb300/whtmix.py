"""Python binding of the WHTMix C ABI (``include/whtmix.h``): argument marshalling only.

Every step of the mixer runs in the CUDA library ``_lib/libwhtmix.so``; this module passes device
pointers, sizes and the current CUDA stream through ctypes, the layer operators' plain calls through a
compiled module that does the same (``_lib/whtmix_torch.so``).  torch supplies device memory and
streams.  There is no CPU path: a missing library or a CPU tensor raises.

The operation (paper Section III-B, Eq. 1-4): Y_b = H_N (G (.) H_N X_b H_C) H_C / (N C) for every
plane X_b [N, C] of X [B, N, C]; the backward returns dX and dG = sum_b (H X_b H)(H dY_b H)/(N C).
"""
from __future__ import annotations

import ctypes
import importlib.machinery
import importlib.util
import os
import threading

import torch
from torch.autograd.function import once_differentiable

from . import build as _build

__all__ = ["forward", "backward", "forward_ex", "backward_ex", "forward_noalloc", "forward_separable",
           "backward_separable",
           "forward_padded", "backward_padded", "project", "block_forward",
           "block_backward", "workspace_bytes", "sync", "plan", "release_workspaces", "WhtmixError", "WHTMixFunction",
           "WHTMixSeparableFunction", "WHTMixBlockFunction", "pad_tokens", "EXPORTS", "library",
           "rms_norm", "rms_norm_backward", "linear", "linear_backward", "quantize_rows", "RMSNormFunction", "LinearFunction",
           "layer_norm", "layer_norm_backward", "gated_linear", "gated_linear_backward", "global_norm", "clip_by_global_norm",
           "LayerNormFunction", "GatedLinearFunction"]

# status codes and dtype codes of include/whtmix.h
OK = 0
STATUS = {0: "OK", 1: "INVALID_ARG", 2: "BAD_SHAPE", 3: "BAD_DTYPE", 4: "MISALIGNED", 5: "ALIAS",
          6: "CUDA", 7: "TIMEOUT", 8: "NO_DEVICE", 9: "WORKSPACE"}
DTYPE_CODE = {torch.float32: 0, torch.bfloat16: 1, torch.int32: 2}
GAIN_DTYPE = {torch.float32: torch.float32, torch.bfloat16: torch.float32, torch.int32: torch.int32}

# every entry point include/whtmix.h declares
EXPORTS = ("whtmix_forward", "whtmix_backward", "whtmix_workspace_bytes", "whtmix_forward_ex",
           "whtmix_backward_ex", "whtmix_sync", "whtmix_release_workspaces", "whtmix_status_string",
           "whtmix_last_cuda_error", "whtmix_plan", "whtmix_forward_noalloc", "whtmix_forward_separable",
           "whtmix_backward_separable", "whtmix_forward_padded", "whtmix_backward_padded", "whtmix_project",
           "whtmix_block_forward", "whtmix_block_backward", "whtmix_forward_x16", "whtmix_rms_norm",
           "whtmix_rms_norm_backward", "whtmix_linear", "whtmix_linear_backward", "whtmix_layer_norm",
           "whtmix_layer_norm_backward", "whtmix_gated_linear", "whtmix_gated_linear_backward", "whtmix_global_norm",
           "whtmix_clip_by_global_norm")

E4M3 = torch.float8_e4m3fn
E4M3_MAX = 448.0
# dtype and activation codes of the layer operators
LAYER_CODE = {torch.float32: 0, torch.bfloat16: 1, E4M3: 3}
ACTIVATION = {"none": 0, "relu": 1, "gelu": 2, "silu": 3}


class WhtmixError(RuntimeError):
    def __init__(self, status: int, what: str):
        self.status = status
        super().__init__(f"{what}: WHTMIX_{'ERR_' if status else ''}{STATUS.get(status, status)} ({status})")


class _Tensor(ctypes.Structure):
    """whtmix_tensor_t"""
    _fields_ = [("in_", ctypes.c_void_p), ("out", ctypes.c_void_p), ("n", ctypes.c_int64), ("dtype", ctypes.c_int)]


_lock = threading.Lock()
_lib = None


def library(path: str | None = None) -> ctypes.CDLL:
    """Load the C library (built by ``__graft_entry__.build()``); raises if it is missing."""
    global _lib
    with _lock:
        if _lib is None:
            path = path or _build.LIB
            if not os.path.exists(path):
                raise RuntimeError(f"WHTMix CUDA library not built ({path}); run __graft_entry__.build()")
            lib = ctypes.CDLL(path)
            i64, p, i, sz = ctypes.c_int64, ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t
            lib.whtmix_forward.argtypes = [p, p, p, i64, i64, i64, i, p]
            lib.whtmix_backward.argtypes = [p, p, p, p, p, i64, i64, i64, i, p]
            lib.whtmix_forward_ex.argtypes = [p, p, p, i64, i64, i64, i, p, sz, p]
            lib.whtmix_forward_noalloc.argtypes = [p, p, p, i64, i64, i64, i, p]
            lib.whtmix_forward_x16.argtypes = [p, p, p, i64, i64, i64, i, p]
            lib.whtmix_backward_ex.argtypes = [p, p, p, p, p, i64, i64, i64, i, p, sz, p]
            lib.whtmix_workspace_bytes.argtypes = [i64, i64, i64, i, i, ctypes.POINTER(sz)]
            lib.whtmix_sync.argtypes = [p]
            lib.whtmix_release_workspaces.argtypes = []
            lib.whtmix_status_string.argtypes = [i]
            lib.whtmix_status_string.restype = ctypes.c_char_p
            lib.whtmix_last_cuda_error.argtypes = []
            lib.whtmix_plan.argtypes = [i64, i64]
            lib.whtmix_forward_separable.argtypes = [p, p, p, p, i64, i64, i64, i64, i, p]
            lib.whtmix_backward_separable.argtypes = [p, p, p, p, p, p, p, i64, i64, i64, i64, i, p]
            lib.whtmix_forward_padded.argtypes = [p, p, p, i64, i64, i64, i64, i, p]
            lib.whtmix_project.argtypes = [p, p, p, i64, i64, i, p]
            lib.whtmix_block_forward.argtypes = [p, p, p, p, p, i64, i64, i64, i, p]
            lib.whtmix_block_backward.argtypes = [p, p, p, p, p, p, p, p, p, i64, i64, i64, i, p]
            lib.whtmix_backward_padded.argtypes = [p, p, p, p, p, i64, i64, i64, i64, i, p]
            f = ctypes.c_float
            lib.whtmix_rms_norm.argtypes = [p] * 6 + [i64] * 6 + [f, i, i, p]
            lib.whtmix_rms_norm_backward.argtypes = [p] * 6 + [i64] * 6 + [f, i, p]
            lib.whtmix_linear.argtypes = [p] * 8 + [i64] * 8 + [i, i, i, p]
            lib.whtmix_linear_backward.argtypes = [p] * 7 + [i64] * 8 + [i, i, p]
            lib.whtmix_layer_norm.argtypes = [p] * 7 + [i64] * 6 + [f, i, i, p]
            lib.whtmix_layer_norm_backward.argtypes = [p] * 7 + [i64] * 6 + [f, i, p]
            lib.whtmix_gated_linear.argtypes = [p] * 7 + [i64] * 7 + [i, i, i, p]
            lib.whtmix_gated_linear_backward.argtypes = [p] * 7 + [i64] * 8 + [i, i, p]
            lib.whtmix_global_norm.argtypes = [p, i64, p, p]
            lib.whtmix_clip_by_global_norm.argtypes = [p, i64, f, p, p]
            for name in EXPORTS:
                if name != "whtmix_status_string":
                    getattr(lib, name).restype = ctypes.c_int
            _lib = lib
    return _lib


_quick = None


def _quick_path():
    """The compiled quick path of the layer operators (csrc/whtmix_torch.cpp): a call with plain tensors and no result
    given runs there; each of its functions returns None for any other call."""
    global _quick
    library()
    with _lock:
        if _quick is None:
            if not os.path.exists(_build.QUICK):
                raise RuntimeError(f"WHTMix binding not built ({_build.QUICK}); run __graft_entry__.build()")
            loader = importlib.machinery.ExtensionFileLoader("whtmix_torch", _build.QUICK)
            module = importlib.util.module_from_spec(importlib.util.spec_from_loader("whtmix_torch", loader))
            loader.exec_module(module)
            module.bind(_check)
            _quick = module
    return _quick


def _check(rc: int, what: str):
    if rc != OK:
        if rc == 6:
            what += f" (cudaError {library().whtmix_last_cuda_error()})"
        raise WhtmixError(rc, what)


def _call(what: str, device: torch.device, stream, fn, *args) -> None:
    """Runs one entry point with ``device`` current, on ``stream`` (default: the device's current
    stream, appended as the last argument); raises WhtmixError on a nonzero status."""
    index = device.index
    if index != torch._C._cuda_getDevice():
        with torch.cuda.device(device):
            return _call(what, device, stream, fn, *args)
    if stream is None:
        # the raw handle: building a Stream object for it takes 2 us, a quarter of a small call
        raw = torch._C._cuda_getCurrentRawStream(index)
    else:
        if stream.device != device:
            raise ValueError(f"stream is on {stream.device}, the tensors on {device}")
        raw = int(stream.cuda_stream)
    rc = fn(*args, raw)
    if rc != OK:
        _check(rc, what)


def _on_device(t: torch.Tensor, device: torch.device, name: str) -> None:
    if not t.is_cuda or t.device != device:
        raise ValueError(f"{name} must be a CUDA tensor on {device} (WHTMix runs on CUDA tensors only)")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")


def _out(t: torch.Tensor | None, shape, dtype: torch.dtype, device: torch.device, name: str) -> torch.Tensor:
    """A result tensor: a new one, or the caller's, checked to be exactly what the library writes
    (the C ABI receives only its pointer)."""
    if t is None:
        return torch.empty(shape, dtype=dtype, device=device)
    if t.dtype != dtype or t.shape != torch.Size(shape):
        raise ValueError(f"{name} must be {dtype} {list(shape)}, got {t.dtype} {list(t.shape)}")
    _on_device(t, device, name)
    return t


def _shape(x: torch.Tensor):
    shape = tuple(x.shape)
    if len(shape) == 3:
        return shape
    if len(shape) != 2:
        raise ValueError("x must be [N, C] or [B, N, C]")
    return (1, *shape)


def _check_tensors(x: torch.Tensor, g: torch.Tensor, *others: torch.Tensor):
    if x.dtype not in DTYPE_CODE:
        raise TypeError(f"unsupported dtype {x.dtype}; expected float32, bfloat16 or int32")
    B, N, C = _shape(x)
    if g.dtype != GAIN_DTYPE[x.dtype]:
        raise TypeError(f"gains must be {GAIN_DTYPE[x.dtype]} for {x.dtype} inputs")
    if tuple(g.shape) != (N, C):
        raise ValueError(f"gains must be [N, C] = [{N}, {C}], got {tuple(g.shape)}")
    device = x.device
    for t in (x, g) + others:
        _on_device(t, device, "every tensor")
    return B, N, C


def forward(x: torch.Tensor, g: torch.Tensor, out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """Y = H_N (G (.) H_N X H_C) H_C / (N C) per plane (unnormalised, mod 2^32, for int32)."""
    B, N, C = _check_tensors(x, g)
    y = _out(out, x.shape, x.dtype, x.device, "out")
    _call("whtmix_forward", x.device, stream, library().whtmix_forward, x.data_ptr(), g.data_ptr(), y.data_ptr(),
          B, N, C, DTYPE_CODE[x.dtype])
    return y


def forward_x16(x: torch.Tensor, g: torch.Tensor, out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """forward whose three-phase kernel rounds the exchanged intermediate plane to bf16 (half the
    workspace traffic; butterflies and gain in fp32); other shapes run exactly as forward."""
    B, N, C = _check_tensors(x, g)
    y = _out(out, x.shape, x.dtype, x.device, "out")
    _call("whtmix_forward_x16", x.device, stream, library().whtmix_forward_x16, x.data_ptr(), g.data_ptr(),
          y.data_ptr(), B, N, C, DTYPE_CODE[x.dtype])
    return y


def forward_noalloc(x: torch.Tensor, g: torch.Tensor, out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """forward without any device allocation: planes of more than 2^22 elements raise WORKSPACE.
    Calls share one fixed scratch array per device, so order them on one stream; make the first
    call on a device outside any stream capture."""
    B, N, C = _check_tensors(x, g)
    y = _out(out, x.shape, x.dtype, x.device, "out")
    _call("whtmix_forward_noalloc", x.device, stream, library().whtmix_forward_noalloc, x.data_ptr(), g.data_ptr(),
          y.data_ptr(), B, N, C, DTYPE_CODE[x.dtype])
    return y


def backward(x: torch.Tensor, g: torch.Tensor, dy: torch.Tensor, dx: torch.Tensor | None = None,
             dg: torch.Tensor | None = None, stream=None):
    """(dX, dG) of the forward map; dG is summed over the batch in ascending order."""
    B, N, C = _check_tensors(x, g, dy)
    if dy.shape != x.shape or dy.dtype != x.dtype:
        raise ValueError("dy must match x in shape and dtype")
    dx = _out(dx, x.shape, x.dtype, x.device, "dx")
    dg = _out(dg, g.shape, g.dtype, x.device, "dg")
    _call("whtmix_backward", x.device, stream, library().whtmix_backward, x.data_ptr(), g.data_ptr(), dy.data_ptr(),
          dx.data_ptr(), dg.data_ptr(), B, N, C, DTYPE_CODE[x.dtype])
    return dx, dg


def _check_log_gains(x: torch.Tensor, g_t: torch.Tensor, g_c: torch.Tensor, *others: torch.Tensor):
    """(B, N_valid, N, C): x holds N_valid tokens per plane, g_t has the padded length N."""
    if x.dtype not in (torch.float32, torch.bfloat16):
        raise TypeError(f"separable gains need float32 or bfloat16 inputs, got {x.dtype}")
    B, n_valid, C = _shape(x)
    if g_t.dtype != torch.float32 or g_c.dtype != torch.float32 or g_t.dim() != 1:
        raise TypeError("log gains must be 1D float32 tensors")
    N = g_t.shape[0]
    if N & (N - 1) or N < max(n_valid, 1):
        raise ValueError(f"g_t must have a power-of-two length >= the {n_valid} tokens of x, got {N}")
    if tuple(g_c.shape) != (C,):
        raise ValueError(f"log gains must be g_t [{N}] and g_c [{C}], got {tuple(g_t.shape)} and {tuple(g_c.shape)}")
    for t in (x, g_t, g_c) + others:
        _on_device(t, x.device, "every tensor")
    return B, n_valid, N, C


def forward_separable(x: torch.Tensor, g_t: torch.Tensor, g_c: torch.Tensor, out: torch.Tensor | None = None,
                      stream=None) -> torch.Tensor:
    """The forward with the paper's log-domain gains (Section III-B, Eq. 2-3):
    G[n, c] = exp(g_t[n]) exp(g_c[c]).  When x has fewer tokens than g_t (not a power of two), the
    planes are zero-padded to len(g_t) tokens inside the library and y keeps x's tokens."""
    B, n_valid, N, C = _check_log_gains(x, g_t, g_c)
    y = _out(out, x.shape, x.dtype, x.device, "out")
    _call("whtmix_forward_separable", x.device, stream, library().whtmix_forward_separable, x.data_ptr(),
          g_t.data_ptr(), g_c.data_ptr(), y.data_ptr(), B, n_valid, N, C, DTYPE_CODE[x.dtype])
    return y


def backward_separable(x: torch.Tensor, g_t: torch.Tensor, g_c: torch.Tensor, dy: torch.Tensor,
                       dx: torch.Tensor | None = None, dg_t: torch.Tensor | None = None,
                       dg_c: torch.Tensor | None = None, stream=None):
    """(dX, dg_t, dg_c) of forward_separable."""
    B, n_valid, N, C = _check_log_gains(x, g_t, g_c, dy)
    if dy.shape != x.shape or dy.dtype != x.dtype:
        raise ValueError("dy must match x in shape and dtype")
    dx = _out(dx, x.shape, x.dtype, x.device, "dx")
    dg_t = _out(dg_t, g_t.shape, g_t.dtype, x.device, "dg_t")
    dg_c = _out(dg_c, g_c.shape, g_c.dtype, x.device, "dg_c")
    _call("whtmix_backward_separable", x.device, stream, library().whtmix_backward_separable, x.data_ptr(),
          g_t.data_ptr(), g_c.data_ptr(), dy.data_ptr(), dx.data_ptr(), dg_t.data_ptr(), dg_c.data_ptr(), B,
          n_valid, N, C, DTYPE_CODE[x.dtype])
    return dx, dg_t, dg_c


def _check_padded(x: torch.Tensor, g: torch.Tensor, *others: torch.Tensor):
    """(B, N_valid, N, C) for a padded call: x holds N_valid tokens, g is the padded [N, C]."""
    if x.dtype not in DTYPE_CODE:
        raise TypeError(f"unsupported dtype {x.dtype}; expected float32, bfloat16 or int32")
    B, n_valid, C = _shape(x)
    if g.dtype != GAIN_DTYPE[x.dtype] or g.dim() != 2 or g.shape[1] != C:
        raise ValueError(f"gains must be {GAIN_DTYPE[x.dtype]} [N, {C}]")
    N = g.shape[0]
    if N & (N - 1) or N < max(n_valid, 1):
        raise ValueError(f"gains must have a power-of-two token count >= the {n_valid} tokens of x, got {N}")
    for t in (x, g) + others:
        _on_device(t, x.device, "every tensor")
    return B, n_valid, N, C


def forward_padded(x: torch.Tensor, g: torch.Tensor, out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """The forward on planes zero-padded from x's N_valid tokens to g's N (a power of two), inside the
    library; y keeps x's N_valid tokens (Section III-B: pad before H_N, discard the padded outputs)."""
    B, n_valid, N, C = _check_padded(x, g)
    y = _out(out, x.shape, x.dtype, x.device, "out")
    _call("whtmix_forward_padded", x.device, stream, library().whtmix_forward_padded, x.data_ptr(), g.data_ptr(),
          y.data_ptr(), B, n_valid, N, C, DTYPE_CODE[x.dtype])
    return y


def backward_padded(x: torch.Tensor, g: torch.Tensor, dy: torch.Tensor, dx: torch.Tensor | None = None,
                    dg: torch.Tensor | None = None, stream=None):
    """(dX, dG) of forward_padded; dX keeps x's tokens, dG is the padded [N, C]."""
    B, n_valid, N, C = _check_padded(x, g, dy)
    if dy.shape != x.shape or dy.dtype != x.dtype:
        raise ValueError("dy must match x in shape and dtype")
    dx = _out(dx, x.shape, x.dtype, x.device, "dx")
    dg = _out(dg, g.shape, g.dtype, x.device, "dg")
    _call("whtmix_backward_padded", x.device, stream, library().whtmix_backward_padded, x.data_ptr(), g.data_ptr(),
          dy.data_ptr(), dx.data_ptr(), dg.data_ptr(), B, n_valid, N, C, DTYPE_CODE[x.dtype])
    return dx, dg


def project(x: torch.Tensor, w: torch.Tensor, out_dtype: torch.dtype = torch.bfloat16,
            out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """z = x w^T per token on the tensor cores (x [..., C] bf16, w [C, C] bf16 as (out, in))."""
    if x.dtype != torch.bfloat16 or w.dtype != torch.bfloat16:
        raise TypeError("project takes bfloat16 x and w")
    if out_dtype not in (torch.float32, torch.bfloat16):
        raise TypeError(f"project writes float32 or bfloat16, not {out_dtype}")
    C = x.shape[-1]
    if tuple(w.shape) != (C, C):
        raise ValueError(f"w must be [{C}, {C}]")
    for t in (x, w):
        _on_device(t, x.device, "x and w")
    z = _out(out, x.shape, out_dtype, x.device, "out")
    _call("whtmix_project", x.device, stream, library().whtmix_project, x.data_ptr(), w.data_ptr(), z.data_ptr(),
          x.numel() // C, C, DTYPE_CODE[out_dtype])
    return z


def block_forward(x: torch.Tensor, w_in: torch.Tensor, g: torch.Tensor, w_out: torch.Tensor,
                  out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """The mixer block of Section III-B, Eq. 1-4: Y = mix(X W_in^T) W_out^T (bf16)."""
    B, N, C = _check_tensors(x, g)
    for t in (w_in, w_out):
        if t.dtype != torch.bfloat16 or tuple(t.shape) != (C, C):
            raise ValueError(f"w_in and w_out must be bfloat16 [{C}, {C}]")
        _on_device(t, x.device, "w_in and w_out")
    y = _out(out, x.shape, x.dtype, x.device, "out")
    _call("whtmix_block_forward", x.device, stream, library().whtmix_block_forward, x.data_ptr(), w_in.data_ptr(),
          g.data_ptr(), w_out.data_ptr(), y.data_ptr(), B, N, C, DTYPE_CODE[x.dtype])
    return y


def block_backward(x: torch.Tensor, w_in: torch.Tensor, g: torch.Tensor, w_out: torch.Tensor, dy: torch.Tensor,
                   dx: torch.Tensor | None = None, dw_in: torch.Tensor | None = None, dg: torch.Tensor | None = None,
                   dw_out: torch.Tensor | None = None, stream=None):
    """(dX, dW_in, dG, dW_out) of block_forward for the upstream gradient dy (bf16); the gain and
    weight gradients are float32."""
    B, N, C = _check_tensors(x, g, dy)
    if dy.shape != x.shape or dy.dtype != x.dtype:
        raise ValueError("dy must match x in shape and dtype")
    for t in (w_in, w_out):
        if t.dtype != torch.bfloat16 or tuple(t.shape) != (C, C):
            raise ValueError(f"w_in and w_out must be bfloat16 [{C}, {C}]")
        _on_device(t, x.device, "w_in and w_out")
    dx = _out(dx, x.shape, x.dtype, x.device, "dx")
    dw_in = _out(dw_in, (C, C), torch.float32, x.device, "dw_in")
    dg = _out(dg, g.shape, torch.float32, x.device, "dg")
    dw_out = _out(dw_out, (C, C), torch.float32, x.device, "dw_out")
    _call("whtmix_block_backward", x.device, stream, library().whtmix_block_backward, x.data_ptr(), w_in.data_ptr(),
          g.data_ptr(), w_out.data_ptr(), dy.data_ptr(), dx.data_ptr(), dw_in.data_ptr(), dg.data_ptr(),
          dw_out.data_ptr(), B, N, C, DTYPE_CODE[x.dtype])
    return dx, dw_in, dg, dw_out


# ---- the layer around the mixer: RMS norm and the matrix product with its epilogue ----

def _rows(t: torch.Tensor, name: str, index: int):
    """(rows, channels, stride) of a tensor [..., C] on CUDA device `index` whose channels are contiguous and whose
    other axes step through memory with one stride (any contiguous tensor, a slice of channels of one, a view of
    every k-th token)."""
    if t.get_device() != index or index < 0:
        raise ValueError(f"{name} must be a CUDA tensor on the first tensor's device (WHTMix runs on CUDA tensors only), "
                         f"it is on {t.device}")
    shape = t.shape
    if not shape or shape[-1] < 1:
        raise ValueError(f"{name} must have at least one channel, got shape {list(shape)}")
    C = shape[-1]
    rows = shape[0] if len(shape) == 2 else t.numel() // C
    if rows == 0 or t.is_contiguous():
        return rows, C, C
    strides = t.stride()
    if C > 1 and strides[-1] != 1:
        raise ValueError(f"{name} must have contiguous channels, got strides {list(strides)}")
    step, expect = 0, 0
    for n, st in zip(reversed(shape[:-1]), reversed(strides[:-1])):
        if n == 1:
            continue
        if step == 0:
            step = st
        elif st != expect:
            raise ValueError(f"the rows of {name} must lie at one stride, got shape {list(shape)}, strides {list(strides)}")
        expect = st * n
    if rows > 1 and step < C:
        raise ValueError(f"the rows of {name} overlap: shape {list(shape)}, strides {list(strides)}")
    return rows, C, step or C


def _vector(t: torch.Tensor, shape, name: str, index: int) -> int:
    """The address of a contiguous float32 tensor of the given shape."""
    if t.dtype != torch.float32 or t.shape != shape:
        raise ValueError(f"{name} must be float32 {list(shape)}, got {t.dtype} {list(t.shape)}")
    if t.get_device() != index or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous CUDA tensor on the first tensor's device")
    return t.data_ptr()


def _stride(t: torch.Tensor, shape, dtype: torch.dtype, name: str, index: int) -> int:
    """The row stride of a row matrix of the given shape and dtype."""
    if t.dtype != dtype or t.shape != shape:
        raise ValueError(f"{name} must be {dtype} {list(shape)}, got {t.dtype} {list(t.shape)}")
    if t.is_contiguous() and t.get_device() == index:
        return shape[-1]
    return _rows(t, name, index)[2]


def _on(stream, device: torch.device):
    """A context in which the call runs on the given stream and results are allocated as that stream's: memory of another
    stream's may still be in use there, and goes back to it, while this one writes."""
    if stream.device != device:
        raise ValueError(f"stream is on {stream.device}, the tensors on {device}")
    return torch.cuda.stream(stream)


def rms_norm(x: torch.Tensor, w: torch.Tensor, residual: torch.Tensor | None = None, eps: float = 1e-6,
             out_dtype: torch.dtype | None = None, out: torch.Tensor | None = None, h: torch.Tensor | None = None,
             scale: torch.Tensor | None = None, stream=None):
    """h = x + residual; y = h w / sqrt(mean(h^2) + eps) over the last axis (x float32 or bfloat16, w float32).

    Returns y, or with out_dtype float8_e4m3fn (values, scales): y = values * scales[..., None], one float32 scale a
    token; with a residual h is appended.  8-bit values that are allocated here have rows at a 16-byte pitch (a view
    of a wider tensor where the last axis is no multiple of 16)."""
    if x.is_cuda and out is None and h is None and scale is None and stream is None:
        done = (_quick or _quick_path()).rms_norm(x, w, residual, eps, out_dtype)
        if done is not None:
            return done
    if stream is not None and x.is_cuda and (out is None or (h is None and residual is not None) or
                                             (scale is None and out_dtype == E4M3)):
        with _on(stream, x.device):
            return rms_norm(x, w, residual, eps, out_dtype, out, h, scale)
    dtype = x.dtype
    if dtype != torch.bfloat16 and dtype != torch.float32:
        raise TypeError(f"rms_norm takes float32 or bfloat16, got {dtype}")
    eight = out_dtype == E4M3
    if not eight and out_dtype is not None and out_dtype != dtype:
        raise TypeError(f"rms_norm of {dtype} writes {dtype} or {E4M3}, not {out_dtype}")
    shape, index = x.shape, x.get_device()
    T, D, xs = _rows(x, "x", index)
    wp = _vector(w, (D,), "w", index)
    device = x.device
    rp = rs = hp = hs = sp = 0
    if residual is not None:
        rs = _stride(residual, shape, dtype, "residual", index)
        rp = residual.data_ptr()
        if h is None:
            h, hs = torch.empty(shape, dtype=dtype, device=device), D
        else:
            hs = _stride(h, shape, dtype, "h", index)
        hp = h.data_ptr()
    elif h is not None:
        raise ValueError("h is the sum of x and the residual: it needs a residual")
    if out is not None:
        ys = _stride(out, shape, E4M3 if eight else dtype, "out", index)
    elif eight and D % 16:
        # rows at a 16-byte pitch, as the tensor cores' loads want them: linear takes them as they lie
        ys = (D + 15) // 16 * 16
        out = torch.empty((*shape[:-1], ys), dtype=E4M3, device=device)[..., :D]
    else:
        out, ys = torch.empty(shape, dtype=E4M3 if eight else dtype, device=device), D
    if eight:
        if scale is None:
            scale = torch.empty(shape[:-1], dtype=torch.float32, device=device)
            sp = scale.data_ptr()
        else:
            sp = _vector(scale, shape[:-1], "scale", index)
    elif scale is not None:
        raise ValueError(f"scale belongs to an output of {E4M3}")
    code = LAYER_CODE[dtype]
    _call("whtmix_rms_norm", device, stream, (_lib or library()).whtmix_rms_norm, x.data_ptr(), rp, wp, hp, out.data_ptr(),
          sp, T, D, xs, rs, hs, ys, eps, code, 3 if eight else code)
    if eight:
        return (out, scale) if residual is None else (out, scale, h)
    return out if residual is None else (out, h)


def rms_norm_backward(h: torch.Tensor, w: torch.Tensor, dy: torch.Tensor, dh: torch.Tensor | None = None,
                      eps: float = 1e-6, dx: torch.Tensor | None = None, dw: torch.Tensor | None = None, stream=None):
    """(dx, dw) of rms_norm from its sum h (x where it had no residual); dh is the gradient that reaches h
    directly.  dx is the gradient of x and of the residual; dw is float32."""
    if h.is_cuda and dx is None and dw is None and stream is None:
        done = (_quick or _quick_path()).rms_norm_backward(h, w, dy, dh, eps)
        if done is not None:
            return done
    if stream is not None and h.is_cuda and (dx is None or dw is None):
        with _on(stream, h.device):
            return rms_norm_backward(h, w, dy, dh, eps, dx, dw)
    dtype = h.dtype
    if dtype != torch.bfloat16 and dtype != torch.float32:
        raise TypeError(f"rms_norm_backward takes float32 or bfloat16, got {dtype}")
    shape, index = h.shape, h.get_device()
    T, D, hs = _rows(h, "h", index)
    wp = _vector(w, (D,), "w", index)
    device = h.device
    dys = _stride(dy, shape, dtype, "dy", index)
    dhs = 0 if dh is None else _stride(dh, shape, dtype, "dh", index)
    if dx is None:
        dx, dxs = torch.empty(shape, dtype=dtype, device=device), D
    else:
        dxs = _stride(dx, shape, dtype, "dx", index)
    if dw is None:
        dw = torch.empty(D, dtype=torch.float32, device=device)
    _call("whtmix_rms_norm_backward", device, stream, (_lib or library()).whtmix_rms_norm_backward, h.data_ptr(), wp,
          dy.data_ptr(), 0 if dh is None else dh.data_ptr(), dx.data_ptr(), _vector(dw, (D,), "dw", index), T, D, hs, dys, dhs,
          dxs, eps, LAYER_CODE[dtype])
    return dx, dw


def _activation(name: str) -> int:
    code = ACTIVATION.get(name)
    if code is None:
        raise ValueError(f"activation must be one of {sorted(ACTIVATION)}, got {name!r}")
    return code


def linear(x: torch.Tensor, w: torch.Tensor, bias: torch.Tensor | None = None, activation: str = "none",
           residual: torch.Tensor | None = None, x_scale: torch.Tensor | None = None,
           w_scale: torch.Tensor | None = None, preact: torch.Tensor | bool | None = None,
           out_dtype: torch.dtype = torch.bfloat16, out: torch.Tensor | None = None, stream=None):
    """y = act(x w^T + bias) + residual over the last axis: x [..., K] and w [N, K] bfloat16, or both float8_e4m3fn
    with float32 scales x_scale [...] and w_scale [N]; bias [N] float32; residual and y [..., N] of out_dtype
    (bfloat16 or float32).  preact=True, or a bfloat16 tensor, also returns the pre-activation: (y, preact)."""
    act = _activation(activation)
    if x.is_cuda and out is None and stream is None and (preact is None or preact.__class__ is bool):
        done = (_quick or _quick_path()).linear(x, w, bias, act, residual, x_scale, w_scale, preact, out_dtype)
        if done is not None:
            return done
    if stream is not None and x.is_cuda and (out is None or preact is True):
        with _on(stream, x.device):
            return linear(x, w, bias, activation, residual, x_scale, w_scale, preact, out_dtype, out)
    dtype, device, index = x.dtype, x.device, x.get_device()
    if dtype != torch.bfloat16 and dtype != E4M3:
        raise TypeError(f"linear takes bfloat16 or {E4M3}, got {dtype}")
    if out_dtype != torch.bfloat16 and out_dtype != torch.float32:
        raise TypeError(f"linear writes bfloat16 or float32, not {out_dtype}")
    N, K = w.shape if w.dim() == 2 else (0, 0)
    if w.dtype != dtype or K != x.shape[-1]:
        raise ValueError(f"w must be {dtype} [N, {x.shape[-1]}], got {w.dtype} {list(w.shape)}")
    T, _, xs = _rows(x, "x", index)
    ws = _rows(w, "w", index)[2]
    lead = x.shape[:-1]
    shape = lead + (N,)
    xsp = wsp = bp = rp = rs = pp = ps = 0
    if dtype == E4M3:
        if x_scale is None or w_scale is None:
            raise ValueError(f"{E4M3} needs x_scale and w_scale")
        xsp, wsp = _vector(x_scale, lead, "x_scale", index), _vector(w_scale, (N,), "w_scale", index)
    elif x_scale is not None or w_scale is not None:
        raise ValueError(f"scales belong to {E4M3} operands")
    if bias is not None:
        bp = _vector(bias, (N,), "bias", index)
    if residual is not None:
        rs = _stride(residual, shape, out_dtype, "residual", index)
        rp = residual.data_ptr()
    save = preact is not None and preact is not False
    if save:
        if out_dtype != torch.bfloat16:
            raise ValueError("preact is bfloat16 and goes with a bfloat16 output")
        if preact is True:
            preact, ps = torch.empty(shape, dtype=torch.bfloat16, device=device), N
        else:
            ps = _stride(preact, shape, torch.bfloat16, "preact", index)
        pp = preact.data_ptr()
    if out is None:
        out, ys = torch.empty(shape, dtype=out_dtype, device=device), N
    else:
        ys = _stride(out, shape, out_dtype, "out", index)
    _call("whtmix_linear", device, stream, (_lib or library()).whtmix_linear, x.data_ptr(), w.data_ptr(), xsp, wsp, bp, rp,
          pp, out.data_ptr(), T, N, K, xs, ws, rs, ps, ys, act, LAYER_CODE[dtype], LAYER_CODE[out_dtype])
    return (out, preact) if save else out


def linear_backward(x: torch.Tensor, w: torch.Tensor, dy: torch.Tensor, p: torch.Tensor | None = None,
                    activation: str = "none", need_dx: bool = True, need_dw: bool = True, need_db: bool = True,
                    dw_dtype: torch.dtype = torch.bfloat16, dx: torch.Tensor | None = None,
                    dw: torch.Tensor | None = None, db: torch.Tensor | None = None, stream=None):
    """(dx, dw, db) of linear for the upstream gradient dy of y (bfloat16), from the stored pre-activation p (needed
    unless the activation is "none"); None in the place of a gradient that is not needed.  The residual's gradient is
    dy itself.  dw is bfloat16 or float32, db float32."""
    act = _activation(activation)
    if x.is_cuda and dx is None and dw is None and db is None and stream is None:
        done = (_quick or _quick_path()).linear_backward(x, w, dy, p, act, need_dx, need_dw, need_db, dw_dtype)
        if done is not None:
            return done
    if stream is not None and x.is_cuda and ((dx is None and need_dx) or (dw is None and need_dw) or (db is None and need_db)):
        with _on(stream, x.device):
            return linear_backward(x, w, dy, p, activation, need_dx, need_dw, need_db, dw_dtype, dx, dw, db)
    device, index = x.device, x.get_device()
    if x.dtype != torch.bfloat16:
        raise TypeError(f"linear_backward takes bfloat16, got {x.dtype}")
    if dw_dtype != torch.bfloat16 and dw_dtype != torch.float32:
        raise TypeError(f"dw is bfloat16 or float32, not {dw_dtype}")
    N, K = w.shape if w.dim() == 2 else (0, 0)
    if w.dtype != torch.bfloat16 or K != x.shape[-1]:
        raise ValueError(f"w must be {torch.bfloat16} [N, {x.shape[-1]}], got {w.dtype} {list(w.shape)}")
    T, _, xs = _rows(x, "x", index)
    ws = _rows(w, "w", index)[2]
    shape = x.shape[:-1] + (N,)
    dys = _stride(dy, shape, torch.bfloat16, "dy", index)
    pp = ps = dxp = dxs = dwp = dbp = 0
    if act:
        if p is None:
            raise ValueError(f"the backward of {activation} needs the pre-activation p")
        ps = _stride(p, shape, torch.bfloat16, "p", index)
        pp = p.data_ptr()
    if dx is not None:
        dxs = _stride(dx, x.shape, torch.bfloat16, "dx", index)
        dxp = dx.data_ptr()
    elif need_dx:
        dx, dxs = torch.empty(x.shape, dtype=torch.bfloat16, device=device), K
        dxp = dx.data_ptr()
    if dw is not None or need_dw:
        dw = _out(dw, (N, K), dw_dtype, device, "dw")
        dwp = dw.data_ptr()
    if db is not None or need_db:
        db = torch.empty(N, dtype=torch.float32, device=device) if db is None else db
        dbp = _vector(db, (N,), "db", index)
    _call("whtmix_linear_backward", device, stream, (_lib or library()).whtmix_linear_backward, x.data_ptr(), w.data_ptr(),
          dy.data_ptr(), pp, dxp, dwp, dbp, T, N, K, xs, ws, dys, ps, dxs, act, LAYER_CODE[dw_dtype])
    return dx, dw, db


def quantize_rows(w: torch.Tensor):
    """(values, scales) of a weight [N, K] in 8 bits, laid out once when it is loaded: values float8_e4m3fn,
    scales [N] float32 = max |row| / 448 (1 for a row of zeros), w = values * scales[:, None] to rounding."""
    w = w.float()
    scale = w.abs().amax(1) / E4M3_MAX
    scale = torch.where(scale == 0, torch.ones_like(scale), scale)
    # (a scale below float32's normal numbers is rounded by more than the type's 464 / 448 allows: 2.1e-42 / 4.2e-45 = 500)
    return (w / scale[:, None]).clamp(-E4M3_MAX, E4M3_MAX).to(E4M3), scale


# ---- layer norm, the gated feed-forward half, clipping of a step's gradients ----

def layer_norm(x: torch.Tensor, w: torch.Tensor, b: torch.Tensor | None = None, residual: torch.Tensor | None = None,
               eps: float = 1e-5, out_dtype: torch.dtype | None = None, out: torch.Tensor | None = None,
               h: torch.Tensor | None = None, scale: torch.Tensor | None = None, stream=None):
    """h = x + residual; y = (h - mean(h)) w / sqrt(var(h) + eps) + b over the last axis (x float32 or bfloat16, w and b
    float32; var without correction).

    Returns, writes and allocates what rms_norm does: y, or with out_dtype float8_e4m3fn (values, scales); with a residual
    h is appended."""
    if x.is_cuda and out is None and h is None and scale is None and stream is None:
        done = (_quick or _quick_path()).layer_norm(x, w, b, residual, eps, out_dtype)
        if done is not None:
            return done
    if stream is not None and x.is_cuda and (out is None or (h is None and residual is not None) or
                                             (scale is None and out_dtype == E4M3)):
        with _on(stream, x.device):
            return layer_norm(x, w, b, residual, eps, out_dtype, out, h, scale)
    dtype = x.dtype
    if dtype != torch.bfloat16 and dtype != torch.float32:
        raise TypeError(f"layer_norm takes float32 or bfloat16, got {dtype}")
    eight = out_dtype == E4M3
    if not eight and out_dtype is not None and out_dtype != dtype:
        raise TypeError(f"layer_norm of {dtype} writes {dtype} or {E4M3}, not {out_dtype}")
    shape, index = x.shape, x.get_device()
    T, D, xs = _rows(x, "x", index)
    wp = _vector(w, (D,), "w", index)
    bp = 0 if b is None else _vector(b, (D,), "b", index)
    device = x.device
    rp = rs = hp = hs = sp = 0
    if residual is not None:
        rs = _stride(residual, shape, dtype, "residual", index)
        rp = residual.data_ptr()
        if h is None:
            h, hs = torch.empty(shape, dtype=dtype, device=device), D
        else:
            hs = _stride(h, shape, dtype, "h", index)
        hp = h.data_ptr()
    elif h is not None:
        raise ValueError("h is the sum of x and the residual: it needs a residual")
    if out is not None:
        ys = _stride(out, shape, E4M3 if eight else dtype, "out", index)
    elif eight and D % 16:
        # rows at a 16-byte pitch, as the tensor cores' loads want them: linear and gated_linear take them as they lie
        ys = (D + 15) // 16 * 16
        out = torch.empty((*shape[:-1], ys), dtype=E4M3, device=device)[..., :D]
    else:
        out, ys = torch.empty(shape, dtype=E4M3 if eight else dtype, device=device), D
    if eight:
        if scale is None:
            scale = torch.empty(shape[:-1], dtype=torch.float32, device=device)
            sp = scale.data_ptr()
        else:
            sp = _vector(scale, shape[:-1], "scale", index)
    elif scale is not None:
        raise ValueError(f"scale belongs to an output of {E4M3}")
    code = LAYER_CODE[dtype]
    _call("whtmix_layer_norm", device, stream, (_lib or library()).whtmix_layer_norm, x.data_ptr(), rp, wp, bp, hp, out.data_ptr(),
          sp, T, D, xs, rs, hs, ys, eps, code, 3 if eight else code)
    if eight:
        return (out, scale) if residual is None else (out, scale, h)
    return out if residual is None else (out, h)


def layer_norm_backward(h: torch.Tensor, w: torch.Tensor, dy: torch.Tensor, dh: torch.Tensor | None = None,
                        eps: float = 1e-5, dx: torch.Tensor | None = None, dw: torch.Tensor | None = None,
                        db: torch.Tensor | None = None, need_db: bool = True, stream=None):
    """(dx, dw, db) of layer_norm from its sum h (x where it had no residual); dh is the gradient that reaches h
    directly.  dx is the gradient of x and of the residual; dw and db are float32, db None where it is not needed."""
    if h.is_cuda and dx is None and dw is None and db is None and stream is None:
        done = (_quick or _quick_path()).layer_norm_backward(h, w, dy, dh, eps, need_db)
        if done is not None:
            return done
    if stream is not None and h.is_cuda and (dx is None or dw is None or (db is None and need_db)):
        with _on(stream, h.device):
            return layer_norm_backward(h, w, dy, dh, eps, dx, dw, db, need_db)
    dtype = h.dtype
    if dtype != torch.bfloat16 and dtype != torch.float32:
        raise TypeError(f"layer_norm_backward takes float32 or bfloat16, got {dtype}")
    shape, index = h.shape, h.get_device()
    T, D, hs = _rows(h, "h", index)
    wp = _vector(w, (D,), "w", index)
    device = h.device
    dys = _stride(dy, shape, dtype, "dy", index)
    dhs = 0 if dh is None else _stride(dh, shape, dtype, "dh", index)
    if dx is None:
        dx, dxs = torch.empty(shape, dtype=dtype, device=device), D
    else:
        dxs = _stride(dx, shape, dtype, "dx", index)
    dw = torch.empty(D, dtype=torch.float32, device=device) if dw is None else dw
    dbp = 0
    if db is not None or need_db:
        db = torch.empty(D, dtype=torch.float32, device=device) if db is None else db
        dbp = _vector(db, (D,), "db", index)
    _call("whtmix_layer_norm_backward", device, stream, (_lib or library()).whtmix_layer_norm_backward, h.data_ptr(), wp,
          dy.data_ptr(), 0 if dh is None else dh.data_ptr(), dx.data_ptr(), _vector(dw, (D,), "dw", index), dbp, T, D, hs, dys,
          dhs, dxs, eps, LAYER_CODE[dtype])
    return dx, dw, db


def _halves(w: torch.Tensor, dtype: torch.dtype, K: int):
    """(N, K) of a gated weight [2 N, K]."""
    rows, cols = w.shape if w.dim() == 2 else (0, 0)
    if w.dtype != dtype or cols != K or rows < 2 or rows % 2:
        raise ValueError(f"w must be {dtype} [2 N, {K}], got {w.dtype} {list(w.shape)}")
    return rows // 2, cols


def gated_linear(x: torch.Tensor, w: torch.Tensor, bias: torch.Tensor | None = None, activation: str = "silu",
                 x_scale: torch.Tensor | None = None, w_scale: torch.Tensor | None = None,
                 preact: torch.Tensor | bool | None = None, out_dtype: torch.dtype = torch.bfloat16,
                 out: torch.Tensor | None = None, stream=None):
    """y = act(x wg^T + bg) (x wu^T + bu) over the last axis, the first half of a gated feed-forward block: x [..., K] and
    w [2 N, K] (N rows wg, then N rows wu) bfloat16, or both float8_e4m3fn with float32 scales x_scale [...] and w_scale
    [2 N]; bias [2 N] float32; y [..., N] of out_dtype (bfloat16 or float32).  preact=True, or a bfloat16 tensor
    [..., 2 N], also returns both pre-activations: (y, preact)."""
    act = _activation(activation)
    if x.is_cuda and out is None and stream is None and (preact is None or preact.__class__ is bool):
        done = (_quick or _quick_path()).gated_linear(x, w, bias, act, x_scale, w_scale, preact, out_dtype)
        if done is not None:
            return done
    if stream is not None and x.is_cuda and (out is None or preact is True):
        with _on(stream, x.device):
            return gated_linear(x, w, bias, activation, x_scale, w_scale, preact, out_dtype, out)
    dtype, device, index = x.dtype, x.device, x.get_device()
    if dtype != torch.bfloat16 and dtype != E4M3:
        raise TypeError(f"gated_linear takes bfloat16 or {E4M3}, got {dtype}")
    if out_dtype != torch.bfloat16 and out_dtype != torch.float32:
        raise TypeError(f"gated_linear writes bfloat16 or float32, not {out_dtype}")
    T, K, xs = _rows(x, "x", index)
    N, _ = _halves(w, dtype, K)
    ws = _rows(w, "w", index)[2]
    lead = x.shape[:-1]
    xsp = wsp = bp = pp = ps = 0
    if dtype == E4M3:
        if x_scale is None or w_scale is None:
            raise ValueError(f"{E4M3} needs x_scale and w_scale")
        xsp, wsp = _vector(x_scale, lead, "x_scale", index), _vector(w_scale, (2 * N,), "w_scale", index)
    elif x_scale is not None or w_scale is not None:
        raise ValueError(f"scales belong to {E4M3} operands")
    if bias is not None:
        bp = _vector(bias, (2 * N,), "bias", index)
    save = preact is not None and preact is not False
    if save:
        if out_dtype != torch.bfloat16:
            raise ValueError("preact is bfloat16 and goes with a bfloat16 output")
        if preact is True:
            preact, ps = torch.empty(lead + (2 * N,), dtype=torch.bfloat16, device=device), 2 * N
        else:
            ps = _stride(preact, lead + (2 * N,), torch.bfloat16, "preact", index)
        pp = preact.data_ptr()
    if out is None:
        out, ys = torch.empty(lead + (N,), dtype=out_dtype, device=device), N
    else:
        ys = _stride(out, lead + (N,), out_dtype, "out", index)
    _call("whtmix_gated_linear", device, stream, (_lib or library()).whtmix_gated_linear, x.data_ptr(), w.data_ptr(), xsp, wsp, bp, pp,
          out.data_ptr(), T, N, K, xs, ws, ps, ys, act, LAYER_CODE[dtype], LAYER_CODE[out_dtype])
    return (out, preact) if save else out


def gated_linear_backward(x: torch.Tensor, w: torch.Tensor, dy: torch.Tensor, p: torch.Tensor, activation: str = "silu",
                          need_dx: bool = True, need_dw: bool = True, need_db: bool = True,
                          dw_dtype: torch.dtype = torch.bfloat16, dx: torch.Tensor | None = None,
                          dw: torch.Tensor | None = None, db: torch.Tensor | None = None, stream=None):
    """(dx, dw, db) of gated_linear for the upstream gradient dy of y (bfloat16), from the stored pre-activations p; None in
    the place of a gradient that is not needed.  dw [2 N, K] is bfloat16 or float32, db [2 N] float32."""
    act = _activation(activation)
    if x.is_cuda and dx is None and dw is None and db is None and stream is None:
        done = (_quick or _quick_path()).gated_linear_backward(x, w, dy, p, act, need_dx, need_dw, need_db, dw_dtype)
        if done is not None:
            return done
    if stream is not None and x.is_cuda and ((dx is None and need_dx) or (dw is None and need_dw) or (db is None and need_db)):
        with _on(stream, x.device):
            return gated_linear_backward(x, w, dy, p, activation, need_dx, need_dw, need_db, dw_dtype, dx, dw, db)
    device, index = x.device, x.get_device()
    if x.dtype != torch.bfloat16:
        raise TypeError(f"gated_linear_backward takes bfloat16, got {x.dtype}")
    if dw_dtype != torch.bfloat16 and dw_dtype != torch.float32:
        raise TypeError(f"dw is bfloat16 or float32, not {dw_dtype}")
    T, K, xs = _rows(x, "x", index)
    N, _ = _halves(w, torch.bfloat16, K)
    ws = _rows(w, "w", index)[2]
    lead = x.shape[:-1]
    dys = _stride(dy, lead + (N,), torch.bfloat16, "dy", index)
    ps = _stride(p, lead + (2 * N,), torch.bfloat16, "p", index)
    dxp = dxs = dwp = dbp = 0
    if dx is not None:
        dxs = _stride(dx, x.shape, torch.bfloat16, "dx", index)
        dxp = dx.data_ptr()
    elif need_dx:
        dx, dxs = torch.empty(x.shape, dtype=torch.bfloat16, device=device), K
        dxp = dx.data_ptr()
    if dw is not None or need_dw:
        dw = _out(dw, (2 * N, K), dw_dtype, device, "dw")
        dwp = dw.data_ptr()
    if db is not None or need_db:
        db = torch.empty(2 * N, dtype=torch.float32, device=device) if db is None else db
        dbp = _vector(db, (2 * N,), "db", index)
    _call("whtmix_gated_linear_backward", device, stream, (_lib or library()).whtmix_gated_linear_backward, x.data_ptr(), w.data_ptr(),
          dy.data_ptr(), p.data_ptr(), dxp, dwp, dbp, T, N, K, xs, ws, dys, ps, dxs, act, LAYER_CODE[dw_dtype])
    return dx, dw, db


def _dense(t: torch.Tensor) -> bool:
    """Whether t's elements are all of one piece of memory, in whatever order of its axes."""
    expect = 1
    for st, n in sorted((st, n) for st, n in zip(t.stride(), t.shape) if n != 1):
        if st != expect:
            return False
        expect *= n
    return True


def _list(tensors, out, device: torch.device):
    """whtmix_tensor_t for each tensor (and the one in its place in out)."""
    entries = (_Tensor * len(tensors))()
    for i, t in enumerate(tensors):
        if t.dtype != torch.float32 and t.dtype != torch.bfloat16:
            raise TypeError(f"the tensors must be float32 or bfloat16, tensors[{i}] is {t.dtype}")
        if not t.is_cuda or t.device != device:
            raise ValueError(f"tensors[{i}] must be a CUDA tensor on the first tensor's device, it is on {t.device}")
        if t.numel() and not _dense(t):
            raise ValueError(f"tensors[{i}] must be dense, got shape {list(t.shape)}, strides {list(t.stride())}")
        e = entries[i]
        e.in_, e.n, e.dtype = t.data_ptr(), t.numel(), LAYER_CODE[t.dtype]
        if out is not None:
            o = out[i]
            if o.dtype != t.dtype or o.shape != t.shape or o.device != device or (t.numel() and o.stride() != t.stride()):
                raise ValueError(f"out[{i}] must be like tensors[{i}]: {t.dtype} {list(t.shape)}, strides {list(t.stride())}, on {device}")
            e.out = o.data_ptr()
    return entries


def _norm_device(tensors) -> torch.device:
    for t in tensors:
        if not isinstance(t, torch.Tensor):
            raise TypeError(f"a list of tensors is needed, got {type(t).__name__} in it")
    if not tensors:
        raise ValueError("the list of tensors is empty: it has no device")
    if not tensors[0].is_cuda:
        raise ValueError(f"tensors[0] must be a CUDA tensor (WHTMix runs on CUDA tensors only), it is on {tensors[0].device}")
    return tensors[0].device


def global_norm(tensors, out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """sqrt(sum of all squares) of a list of float32 and bfloat16 tensors on one device, a float32 tensor without axes."""
    if not isinstance(tensors, (list, tuple)):
        tensors = list(tensors)
    if out is None and stream is None:
        done = (_quick or _quick_path()).global_norm(tensors)
        if done is not None:
            return done
    tensors = list(tensors)
    device = _norm_device(tensors)
    if stream is not None and out is None:
        with _on(stream, device):
            return global_norm(tensors)
    entries = _list(tensors, None, device)
    out = _out(out, (), torch.float32, device, "out")
    _call("whtmix_global_norm", device, stream, (_lib or library()).whtmix_global_norm, entries, len(tensors), out.data_ptr())
    return out


def clip_by_global_norm(tensors, max_norm: float, out=None, norm: torch.Tensor | None = None, stream=None):
    """(out, norm): each tensor of the list times min(1, max_norm / (norm + 1e-6)), norm = global_norm(tensors).

    out is a list of tensors like the given ones; with out=tensors they are scaled in place."""
    if not isinstance(tensors, (list, tuple)):
        tensors = list(tensors)
    max_norm = float(max_norm)
    if norm is None and stream is None:
        done = (_quick or _quick_path()).clip_by_global_norm(tensors, max_norm, out)
        if done is not None:
            return done
    tensors = list(tensors)
    device = _norm_device(tensors)
    if out is not None:
        out = list(out)
        if len(out) != len(tensors):
            raise ValueError(f"out must have a tensor for each of the {len(tensors)}, got {len(out)}")
    if not max_norm >= 0:
        raise ValueError(f"max_norm must not be negative, got {max_norm}")
    if stream is not None and (norm is None or out is None):
        with _on(stream, device):
            return clip_by_global_norm(tensors, max_norm, out, norm)
    out = [torch.empty_like(t) for t in tensors] if out is None else out
    entries = _list(tensors, out, device)
    norm = _out(norm, (), torch.float32, device, "norm")
    _call("whtmix_clip_by_global_norm", device, stream, (_lib or library()).whtmix_clip_by_global_norm, entries, len(tensors), max_norm,
          norm.data_ptr())
    return out, norm


def workspace_bytes(B: int, N: int, C: int, dtype: torch.dtype, backward: bool = False) -> int:
    out = ctypes.c_size_t(0)
    _check(library().whtmix_workspace_bytes(B, N, C, DTYPE_CODE[dtype], int(backward), ctypes.byref(out)),
           "whtmix_workspace_bytes")
    return out.value


def forward_ex(x, g, workspace: torch.Tensor, out=None, stream=None):
    """forward with a caller-owned workspace of at least workspace_bytes(...) bytes."""
    B, N, C = _check_tensors(x, g, workspace)
    y = _out(out, x.shape, x.dtype, x.device, "out")
    _call("whtmix_forward_ex", x.device, stream, library().whtmix_forward_ex, x.data_ptr(), g.data_ptr(),
          y.data_ptr(), B, N, C, DTYPE_CODE[x.dtype], workspace.data_ptr(),
          workspace.numel() * workspace.element_size())
    return y


def backward_ex(x, g, dy, workspace: torch.Tensor, dx=None, dg=None, stream=None):
    """backward with a caller-owned workspace of at least workspace_bytes(..., backward=True) bytes."""
    B, N, C = _check_tensors(x, g, dy, workspace)
    if dy.shape != x.shape or dy.dtype != x.dtype:
        raise ValueError("dy must match x in shape and dtype")
    dx = _out(dx, x.shape, x.dtype, x.device, "dx")
    dg = _out(dg, g.shape, g.dtype, x.device, "dg")
    _call("whtmix_backward_ex", x.device, stream, library().whtmix_backward_ex, x.data_ptr(), g.data_ptr(),
          dy.data_ptr(), dx.data_ptr(), dg.data_ptr(), B, N, C, DTYPE_CODE[x.dtype], workspace.data_ptr(),
          workspace.numel() * workspace.element_size())
    return dx, dg


def sync(stream=None) -> None:
    """Synchronise the stream and raise if a device-side bounded wait expired."""
    s = stream if stream is not None else torch.cuda.current_stream()
    _call("whtmix_sync", s.device, s, library().whtmix_sync)


def release_workspaces() -> None:
    _check(library().whtmix_release_workspaces(), "whtmix_release_workspaces")


def plan(N: int, C: int) -> int:
    return library().whtmix_plan(N, C)


def pad_tokens(x: torch.Tensor, n_pad: int | None = None) -> torch.Tensor:
    """Zero-pads the token axis (dim -2) to ``n_pad`` tokens (default: the next power of two, at
    least 1), as the paper does before H_N (Section III-B).  Crop the mixer's output back with
    ``y[..., :n, :]``."""
    n = x.shape[-2]
    target = (1 << max(n - 1, 0).bit_length()) if n_pad is None else n_pad
    if target < max(n, 1) or target & (target - 1):
        raise ValueError(f"n_pad must be a power of two >= the {n} tokens of x, got {target}")
    if target == n:
        return x.contiguous()
    pad = torch.zeros(*x.shape[:-2], target - n, x.shape[-1], dtype=x.dtype, device=x.device)
    return torch.cat([x, pad], dim=-2).contiguous()


class WHTMixFunction(torch.autograd.Function):
    """autograd wrapper: forward and backward both run in the CUDA library."""

    @staticmethod
    def forward(ctx, x, g):
        x, g = x.contiguous(), g.contiguous()
        ctx.save_for_backward(x, g)
        return forward(x, g)

    @staticmethod
    def backward(ctx, dy):
        x, g = ctx.saved_tensors
        dx, dg = backward(x, g, dy.contiguous())
        return dx, dg


class WHTMixSeparableFunction(torch.autograd.Function):
    """autograd wrapper for the log-domain gains: forward and backward both run in the CUDA library."""

    @staticmethod
    def forward(ctx, x, g_t, g_c):
        x, g_t, g_c = x.contiguous(), g_t.contiguous(), g_c.contiguous()
        ctx.save_for_backward(x, g_t, g_c)
        return forward_separable(x, g_t, g_c)

    @staticmethod
    def backward(ctx, dy):
        x, g_t, g_c = ctx.saved_tensors
        return backward_separable(x, g_t, g_c, dy.contiguous())


class WHTMixBlockFunction(torch.autograd.Function):
    """autograd wrapper of the whole block (W_in, mixer, W_out): forward and backward both run in
    the CUDA library; the weight and gain gradients come back in float32."""

    @staticmethod
    def forward(ctx, x, w_in, g, w_out):
        x, w_in, g, w_out = x.contiguous(), w_in.contiguous(), g.contiguous(), w_out.contiguous()
        ctx.save_for_backward(x, w_in, g, w_out)
        return block_forward(x, w_in, g, w_out)

    @staticmethod
    def backward(ctx, dy):
        x, w_in, g, w_out = ctx.saved_tensors
        dx, dw_in, dg, dw_out = block_backward(x, w_in, g, w_out, dy.contiguous())
        return dx, dw_in.to(w_in.dtype), dg, dw_out.to(w_out.dtype)


class RMSNormFunction(torch.autograd.Function):
    """autograd wrapper of rms_norm: (x, w, residual, eps) -> (y, h), h = x where there is no residual."""

    @staticmethod
    def forward(ctx, x, w, residual=None, eps=1e-6):
        if residual is None:
            y, h = rms_norm(x, w, eps=eps), x
        else:
            y, h = rms_norm(x, w, residual=residual, eps=eps)
        ctx.save_for_backward(h, w)
        ctx.eps, ctx.with_residual = eps, residual is not None
        ctx.set_materialize_grads(False)  # where h (or y) is not used, no zeros are filled in and read as its gradient
        return y, h

    @staticmethod
    @once_differentiable
    def backward(ctx, dy, dh):
        h, w = ctx.saved_tensors
        if dy is None:
            dx, dw = dh, None if dh is None else torch.zeros_like(w)
        else:
            dx, dw = rms_norm_backward(h, w, dy.contiguous(), dh=None if dh is None else dh.contiguous(), eps=ctx.eps)
        return dx, dw, dx if ctx.with_residual else None, None


class LinearFunction(torch.autograd.Function):
    """autograd wrapper of linear in bfloat16: (x, w, bias, residual, activation) -> y; dw comes in bfloat16."""

    @staticmethod
    def forward(ctx, x, w, bias=None, residual=None, activation="none"):
        p = None
        if activation == "none":
            y = linear(x, w, bias, residual=residual)
        else:
            y, p = linear(x, w, bias, activation, residual, preact=True)
        ctx.save_for_backward(x, w, p)
        ctx.activation, ctx.with_bias, ctx.with_residual = activation, bias is not None, residual is not None
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        x, w, p = ctx.saved_tensors
        dy = dy.contiguous()
        need = ctx.needs_input_grad
        dx = dw = db = None
        if need[0] or need[1] or (ctx.with_bias and need[2]):
            dx, dw, db = linear_backward(x, w, dy, p, ctx.activation, need_dx=need[0], need_dw=need[1],
                                         need_db=ctx.with_bias and need[2])
        return dx, dw, db, dy if ctx.with_residual else None, None


class LayerNormFunction(torch.autograd.Function):
    """autograd wrapper of layer_norm: (x, w, b, residual, eps) -> (y, h), h = x where there is no residual."""

    @staticmethod
    def forward(ctx, x, w, b=None, residual=None, eps=1e-5):
        if residual is None:
            y, h = layer_norm(x, w, b, eps=eps), x
        else:
            y, h = layer_norm(x, w, b, residual=residual, eps=eps)
        ctx.save_for_backward(h, w)
        ctx.eps, ctx.with_b, ctx.with_residual = eps, b is not None, residual is not None
        ctx.set_materialize_grads(False)  # where h (or y) is not used, no zeros are filled in and read as its gradient
        return y, h

    @staticmethod
    @once_differentiable
    def backward(ctx, dy, dh):
        h, w = ctx.saved_tensors
        if dy is None:
            dx, dw = dh, None if dh is None else torch.zeros_like(w)
            db = torch.zeros_like(dw) if ctx.with_b and dw is not None else None
        else:
            dx, dw, db = layer_norm_backward(h, w, dy.contiguous(), dh=None if dh is None else dh.contiguous(), eps=ctx.eps,
                                             need_db=ctx.with_b)
        return dx, dw, db, dx if ctx.with_residual else None, None


class GatedLinearFunction(torch.autograd.Function):
    """autograd wrapper of gated_linear in bfloat16: (x, w, bias, activation) -> y; dw comes in bfloat16."""

    @staticmethod
    def forward(ctx, x, w, bias=None, activation="silu"):
        y, p = gated_linear(x, w, bias, activation, preact=True)
        ctx.save_for_backward(x, w, p)
        ctx.activation, ctx.with_bias = activation, bias is not None
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        x, w, p = ctx.saved_tensors
        need = ctx.needs_input_grad
        dx = dw = db = None
        if need[0] or need[1] or (ctx.with_bias and need[2]):
            dx, dw, db = gated_linear_backward(x, w, dy.contiguous(), p, ctx.activation, need_dx=need[0], need_dw=need[1],
                                               need_db=ctx.with_bias and need[2])
        return dx, dw, db, None
