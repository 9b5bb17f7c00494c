"""The choice of kernels of the 4-bit products (csrc/mx_choice.h, compiled for the host): every kernel is
reached, sizes at the rule's edges, and the GPU tests' sizes among them."""
from __future__ import annotations

import ctypes
import subprocess
import tempfile
from pathlib import Path

import pytest

from block_sizes import INSIDE, OUTSIDE, PRODUCTS, SKINNY, TILE64, TILE128, TILE256

CSRC = Path(__file__).resolve().parent.parent / "paper_2609_22441_amd" / "csrc"

SHIM = """#include "mx_choice.h"
extern "C" int product(int64_t m, int64_t n, int64_t k) { return ccj::mx_product_choice(m, n, k); }
extern "C" int inside(int64_t m, int64_t n, int64_t k) { return ccj::mx_quantize_inside(m, n, k); }
extern "C" int64_t lds(int64_t m, int64_t k) { return ccj::mx_quantize_lds(m, k); }
"""


def padded(k):
    return -(-k // 128) * 128


@pytest.fixture(scope="module")
def choice():
    with tempfile.TemporaryDirectory() as d:
        src, out = Path(d) / "choice.cpp", Path(d) / "choice.so"
        src.write_text(SHIM)
        subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-shared", "-fPIC", f"-I{CSRC}",
                        str(src), "-o", str(out)], check=True)
        lib = ctypes.CDLL(str(out))
    for name in ("product", "inside"):
        getattr(lib, name).argtypes = [ctypes.c_int64] * 3
    lib.lds.argtypes, lib.lds.restype = [ctypes.c_int64] * 2, ctypes.c_int64
    return lib


@pytest.mark.parametrize("m,n,k,want", [
    (1, 1, 0, SKINNY), (1, 4_096, 4_096, SKINNY), (16, 8_192, 1 << 24, SKINNY), (16, 8_193, 128, TILE64),
    (512, 4_096, 16_384, TILE64), (513, 4_096, 16_384, TILE128), (333, 1_030, 2_176, TILE64),
    (4_096, 4_096, 1_024, TILE256), (4_300, 4_100, 8_192, TILE128), (50_000, 2_048, 2_048, TILE128),
    (50_000, 2_048, 8_192, TILE256), (50_000, 512, 128, TILE256), (1_024, 8_192, 16_384, TILE128),
    (16_384, 8_192, 8_192, TILE256), (2_147_483_647, 2_147_483_647, 4_096, TILE256)])
def test_product(choice, m, n, k, want):
    assert choice.product(m, n, k) == want


@pytest.mark.parametrize("m,n,k,kernel", PRODUCTS)
def test_sizes_of_the_gpu_tests(choice, m, n, k, kernel):
    assert choice.product(m, n, padded(k)) == kernel


def test_every_kernel_is_reached():
    assert {p[3] for p in PRODUCTS} == set(range(4))


def test_where_a_linear_layer_quantises(choice):
    assert all(choice.inside(m, n, padded(k)) for m, n, k in INSIDE)
    assert not any(choice.inside(m, n, padded(k)) for m, n, k in OUTSIDE)


def test_quantised_rows_fit_in_lds(choice):
    """The most values that the rule admits, in as many rows as it does: within what is left of 64 KiB."""
    for m in range(1, 17):
        k = 32_768 // m // 128 * 128
        assert choice.inside(m, 16, k) and choice.lds(m, k) <= 48 << 10
