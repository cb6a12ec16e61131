"""Builds the C-ABI shared library ``_lib/libwhtmix.so`` with nvcc for sm_103a (no torch involved), and where torch is
installed the Python binding's quick path ``_lib/whtmix_torch.so`` (host code, which links to it and to torch).

Usage: ``python -m paper_2607_25234_gb300.build`` (or ``__graft_entry__.build()``).
"""
from __future__ import annotations

import importlib.util
import os
import shutil
import subprocess
import sys
import sysconfig

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(ROOT, "include")
LIBDIR = os.path.join(PKG, "_lib")
LIB = os.path.join(LIBDIR, "libwhtmix.so")
QUICK = os.path.join(LIBDIR, "whtmix_torch.so")
QUICK_SOURCE = "whtmix_torch.cpp"
SOURCES = ["whtmix_capi.cu", "whtmix_fast_f32.cu", "whtmix_fast_bf16.cu", "whtmix_fast_sep_f32.cu", "whtmix_block.cu", "whtmix_plane.cu", "whtmix_small.cu",
           "whtmix_fast_sep_bf16.cu", "whtmix_fast_x16.cu", "whtmix_noalloc.cu", "whtmix_proj.cu", "whtmix_block_bwd.cu",
           "whtmix_layer.cu", "whtmix_norm.cu", "whtmix_linear.cu", "whtmix_gemm_fwd.cu", "whtmix_gemm_e4m3.cu",
           "whtmix_gemm_four.cu", "whtmix_gemm_e4m3_four.cu", "whtmix_gemm_dx.cu", "whtmix_gemm_dw.cu",
           "whtmix_few.cu", "whtmix_gemm_dp.cu", "whtmix_layer_norm.cu", "whtmix_gated.cu", "whtmix_gemm_gated.cu",
           "whtmix_gemm_gated_e4m3.cu", "whtmix_gemm_gated_dp.cu", "whtmix_clip.cu"]
OBJDIR = os.path.join(LIBDIR, "obj")
ARCH = "-gencode=arch=compute_103a,code=sm_103a"


def nvcc() -> str:
    for cand in (os.environ.get("NVCC"), shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found: the WHTMix CUDA library cannot be built")


def _deps() -> list[str]:
    files = [os.path.join(INCLUDE, "whtmix.h")]
    for f in os.listdir(CSRC):
        if f.endswith((".cu", ".cuh", ".h", ".cpp")):
            files.append(os.path.join(CSRC, f))
    return files


def up_to_date() -> bool:
    made = [LIB] if _torch_dir() is None else [LIB, QUICK]
    if not all(os.path.exists(f) for f in made):
        return False
    t = min(os.path.getmtime(f) for f in made)
    return all(os.path.getmtime(f) <= t for f in _deps())


def _torch_dir() -> str | None:
    spec = importlib.util.find_spec("torch")
    return None if spec is None or spec.origin is None else os.path.dirname(spec.origin)


def build(force: bool = False, verbose: bool = False) -> str:
    """Compiles every translation unit in parallel (one nvcc per file), then links the two libraries."""
    if not force and up_to_date():
        return LIB
    os.makedirs(OBJDIR, exist_ok=True)
    common = [nvcc(), ARCH, "-O3", "-lineinfo", "-std=c++17", "-Xcompiler", "-fPIC",
              "-Xcompiler", "-fvisibility=hidden", "-I", INCLUDE, "-I", CSRC]
    if verbose:
        common += ["-Xptxas", "-v"]
    procs, objs = [], []
    for src in SOURCES:
        obj = os.path.join(OBJDIR, src.replace(".cu", f".{os.getpid()}.o"))
        objs.append(obj)
        procs.append((src, subprocess.Popen(common + ["-c", os.path.join(CSRC, src), "-o", obj])))
    torch_dir, quick_obj, quick = _torch_dir(), os.path.join(OBJDIR, f"whtmix_torch.{os.getpid()}.o"), None
    if torch_dir is not None:
        quick = subprocess.Popen(
            [nvcc(), "-O2", "-std=c++17", "-Xcompiler", "-fPIC", "-Xcompiler", "-fvisibility=hidden", "-I", INCLUDE,
             "-isystem", os.path.join(torch_dir, "include"), "-isystem", sysconfig.get_paths()["include"],
             "-c", os.path.join(CSRC, QUICK_SOURCE), "-o", quick_obj])
    failed = [src for src, p in procs if p.wait() != 0]
    quick_failed = quick is not None and quick.wait() != 0
    if failed:
        raise RuntimeError(f"nvcc failed for {failed}")
    tmp = LIB + f".tmp{os.getpid()}"
    subprocess.run([nvcc(), ARCH, "-shared", "-o", tmp] + objs + ["-lcudart"], check=True)
    os.replace(tmp, LIB)
    for obj in objs:
        os.remove(obj)
    if quick is None:
        return LIB
    if quick_failed:
        raise RuntimeError(f"nvcc failed for {QUICK_SOURCE}")
    # both names found beside the module, whose own run path leads there, and in torch's folder
    subprocess.run([nvcc(), "-shared", "-o", tmp, quick_obj, "-L", LIBDIR, "-lwhtmix", "-L", os.path.join(torch_dir, "lib"),
                    "-ltorch_python", "-ltorch_cpu", "-lc10", "-lc10_cuda", "-Xlinker", "-rpath,$ORIGIN",
                    "-Xlinker", "-rpath," + os.path.join(torch_dir, "lib")], check=True)
    os.replace(tmp, QUICK)
    os.remove(quick_obj)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
