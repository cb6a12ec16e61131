"""What the layer operators do on the host at the ends of their ranges, and orderings that no run shows to be missing (CPU)."""
import importlib.util
import os
import re

import pytest
import torch

from paper_2607_25234_gb300 import build as libbuild
from paper_2607_25234_gb300 import whtmix
from test_ordering_host import functions, read


@pytest.fixture(scope="module")
def lib():
    libbuild.build()
    return whtmix.library()


def test_nothing_is_asked_of_an_empty_batch(lib):
    """The gradient of no rows has no address: with dx alone there is nothing to do, with rows there is nothing to write to."""
    def call(T, act=0, dtype=1):
        return lib.whtmix_linear_backward(None, None, None, None, None, None, None, T, 8, 16, 16, 16, 8, 8, 16, act, dtype, None)
    assert call(0) == 0 and call(0, act=2) == 0
    assert call(4) == 1
    assert call(0, act=9) == 1 and call(0, dtype=3) == 3 and call(-1) == 1


LANDED = re.compile(r"(\)\s*)?for \(\w+ j = \w+ > S \? \w+ - S : 0;[^)]*?j < \w+; \+\+j\)\s*(?:if \(!)?tma::wait\(&(?:bars\.)?full\[j % S\]")
COMPLETED = re.compile(r"mma_commit\(&(?:bars\.)?dfull\b(?:(?!warp [<>=]|else if).)*?tma::wait\(&(?:bars\.)?dfull\b", re.S)


def waits_before_it_ends(kernel):
    """The loading warp waits for its last copies whether or not a wait has given up, the warp that issues the products for the last of
    them (a wait of another warp may give up earlier)."""
    landed = LANDED.search(kernel)
    return bool(landed and not landed.group(1)) and bool(COMPLETED.search(kernel))


@pytest.mark.parametrize("name,kernel", [("whtmix_few.cu", "k_few"), ("whtmix_gemm.cuh", "k_gemm"), ("whtmix_gemm_dp.cu", "k_dx_dp")])
def test_copies_and_products_in_flight_are_waited_for_whichever_wait_gave_up(name, kernel):
    text = dict(functions(read(name)))[kernel]
    assert waits_before_it_ends(text)
    # and the check sees one that is missing
    only_then = LANDED.sub(lambda m: "if (bad) " + m.group(0), text)
    assert not waits_before_it_ends(only_then)
    last = [m.end() for m in re.finditer(r"mma_commit\(&(?:bars\.)?dfull\b[^;]*;", text)][-1]
    issuer = text[last:].split("else if" if "else if (warp >=" in text[last:] else "float* sums", 1)[0]
    assert not waits_before_it_ends(text.replace(issuer, issuer.replace("tma::wait", "no_wait")))


@pytest.mark.parametrize("with_torch", [False, True])
def test_the_c_library_is_built_without_torch(tmp_path, monkeypatch, with_torch):
    """With a compiler that only makes its output file and writes down what it was asked."""
    nvcc, log = tmp_path / "nvcc", tmp_path / "log"
    nvcc.write_text('#!/bin/sh\necho "$@" >> ' + str(log) + '\nwhile [ "$1" != -o ]; do shift; done\n: > "$2"\n')
    nvcc.chmod(0o755)
    monkeypatch.setenv("NVCC", str(nvcc))
    for name, value in (("LIBDIR", tmp_path / "lib"), ("OBJDIR", tmp_path / "lib" / "obj"), ("LIB", tmp_path / "lib" / "libwhtmix.so"),
                        ("QUICK", tmp_path / "lib" / "whtmix_torch.so")):
        monkeypatch.setattr(libbuild, name, str(value))
    if not with_torch:
        find = importlib.util.find_spec
        monkeypatch.setattr(importlib.util, "find_spec", lambda name, *a: None if name == "torch" else find(name, *a))
    assert not libbuild.up_to_date()
    assert libbuild.build() == libbuild.LIB and os.path.exists(libbuild.LIB)
    assert os.path.exists(libbuild.QUICK) == with_torch and libbuild.up_to_date()
    assert os.listdir(libbuild.OBJDIR) == []
    for line in log.read_text().splitlines():
        assert with_torch or "torch" not in line.replace(str(tmp_path), "")


@pytest.mark.parametrize("top", [1.0, 1e-30, 9.3e-41, 2.1e-42, 6e-43, 1e-43, 3e38])
def test_rows_of_any_size_have_finite_eight_bit_values(top):
    """Weights of a row whose scale is a float32 below the normal numbers (steps of 2^-149): within a step of 448, no NaN."""
    q, s = whtmix.quantize_rows(torch.tensor([[top, top / 2, -top, 0.0]]))
    v = q.double() * s.double()[:, None]
    w = torch.tensor([[top, top / 2, -top, 0.0]]).double()
    assert bool(torch.isfinite(q.float()).all())
    # the scale is the nearest float32, whose step times 448 is what the largest value may be off by
    assert bool(((v - w).abs() <= 2.0 ** -4 * w.abs() + 448 * 2.0 ** -149).all())
    bad, _ = whtmix.quantize_rows(torch.tensor([[float("nan"), 1.0]]))
    assert bool(torch.isnan(bad.float()).any())
