"""The 8-bit product's choice of kernel (csrc/i8_choice.h, compiled for the host): every kernel is
reached, sizes at the rule's edges, and the GPU tests' sizes among them."""
from __future__ import annotations

import ctypes
import subprocess
import tempfile
from pathlib import Path

import pytest

CSRC = Path(__file__).resolve().parent.parent / "paper_2609_22441_amd" / "csrc"
SKINNY, TILE64, TILE128X64, TILE128_SPLIT, TILE128, TILE256, SHORT = range(7)

SHIM = """#include "i8_choice.h"
extern "C" int product(int64_t m, int64_t n, int64_t k) { return ccj::product_choice(m, n, k); }
extern "C" int skinny(int64_t m, int64_t n, int64_t k) { return ccj::quantize_inside(m, n, k); }
extern "C" int tile(int64_t m, int64_t n, int64_t k) { return ccj::quantize_in_tile(m, n, k); }
"""


@pytest.fixture(scope="module")
def choice():
    with tempfile.TemporaryDirectory() as d:
        src, out = Path(d) / "choice.cpp", Path(d) / "choice.so"
        src.write_text(SHIM)
        subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-shared", "-fPIC", f"-I{CSRC}",
                        str(src), "-o", str(out)], check=True)
        lib = ctypes.CDLL(str(out))
    for name in ("product", "skinny", "tile"):
        getattr(lib, name).argtypes = [ctypes.c_int64] * 3
    return lib


@pytest.mark.parametrize("m,n,k,want", [
    (1, 4_096, 4_096, SKINNY), (16, 4_096, 131_056, SKINNY), (17, 4_096, 2_048, SKINNY),
    (17, 4_096, 2_064, TILE64), (32, 4_096, 2_048, SKINNY), (33, 4_096, 2_048, TILE64),
    (333, 1_030, 2_064, TILE64), (1_024, 1_024, 512, TILE64), (1_025, 1_024, 512, TILE128X64),
    (2_048, 1_024, 8_192, TILE128X64), (2_049, 1_024, 8_192, TILE128_SPLIT),
    (2_049, 1_024, 1_008, TILE128), (4_096, 1_024, 96, TILE128),
    (4_097, 1_024, 96, SHORT), (50_000, 512, 128, SHORT), (50_000, 512, 144, TILE128),
    (1_024, 8_192, 8_192, TILE128), (2_048, 8_192, 8_192, TILE256), (16_384, 8_192, 8_192, TILE256),
    (2_147_483_647, 2_147_483_647, 4_096, TILE256),
])
def test_product(choice, m, n, k, want):
    assert choice.product(m, n, k) == want


@pytest.mark.parametrize("m,n,k,skinny,tile", [
    (1, 4_096, 4_096, True, False), (16, 4_096, 4_080, True, False), (16, 4_096, 4_096, False, False),
    (17, 64, 96, False, True), (1, 16_384, 96, True, False), (1, 16_385, 96, False, False),
    (50_000, 128, 128, False, True), (50_000, 129, 128, False, False),
    (50_000, 128, 144, False, False),
])
def test_where_a_linear_layer_quantises(choice, m, n, k, skinny, tile):
    assert bool(choice.skinny(m, n, k)) == skinny
    if not skinny:
        assert bool(choice.tile(m, n, k)) == tile
