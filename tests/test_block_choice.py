"""The choice of kernels of the 4-bit products (csrc/mx_choice.h) and of the block norms
(csrc/norm_choice.h), compiled for the host: every kernel is reached, sizes at the rule's edges, and the GPU
tests' sizes among them."""
from __future__ import annotations

import ctypes
import subprocess
import tempfile
from pathlib import Path

import pytest

from block_sizes import (INSIDE, MANY_ROWS, NORMS, OUTSIDE, PRODUCTS, SKINNY, TILE64, TILE128,
                         TILE256)

CSRC = Path(__file__).resolve().parent.parent / "paper_2609_22441_amd" / "csrc"

SHIM = """#include "mx_choice.h"
#include "norm_choice.h"
extern "C" int norm(int32_t cols) { return ccj::norm_shape(cols).lanes * 4 + ccj::norm_shape(cols).blocks; }
extern "C" int grad(int32_t cols) {
    return ccj::norm_grad_shape(cols, false).lanes * 4 + ccj::norm_grad_shape(cols, false).blocks;
}
extern "C" int wide_grad(int32_t cols) {
    return ccj::norm_grad_shape(cols, true).lanes * 4 + ccj::norm_grad_shape(cols, true).blocks;
}
extern "C" int64_t groups(int64_t rows, int32_t threads) { return ccj::norm_groups(rows, threads); }
extern "C" int64_t grad_groups(int64_t rows, int32_t cols) {
    return ccj::norm_grad_groups(rows, cols, false);
}
extern "C" int64_t wide_grad_groups(int64_t rows, int32_t cols) {
    return ccj::norm_grad_groups(rows, cols, true);
}
extern "C" int64_t strips(int64_t rows, int32_t cols) { return ccj::norm_wide_strips(rows, cols); }
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
    for name in ("groups", "grad_groups", "wide_grad_groups", "strips"):
        f = getattr(lib, name)
        f.argtypes, f.restype = [ctypes.c_int64, ctypes.c_int32], ctypes.c_int64
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


def kernel(of, cols, any_lanes=True):
    """Lanes and blocks of a kernel: beyond a wavefront some take any number up to 256, 512 or 1,024."""
    lanes, blocks = divmod(of(cols), 4)
    if any_lanes and lanes > 64:
        lanes = min(m for m in (256, 512, 1_024) if lanes <= m)
    return lanes, blocks


def kernels(of, any_lanes=True):
    return {kernel(of, cols, any_lanes) for cols in range(1, 20_000)}


def test_norm_shapes_hold_their_rows(choice):
    """A row's lanes hold all of its blocks, and no fewer lanes of the same kernel would."""
    for cols in list(range(1, 16_385)) + [16_385, 1 << 24]:
        for of, most in ((choice.norm, 16_384), (choice.grad, 8_192), (choice.wide_grad, 8_192)):
            lanes, blocks = divmod(of(cols), 4)
            assert (lanes == 0) == (cols > most)
            assert lanes == 0 or lanes * blocks * 8 >= cols


def test_the_gpu_tests_reach_every_norm_kernel(choice):
    """Of each kernel, rows of whole blocks and others; and more rows than a launch goes through at once."""
    for of, any_lanes in ((choice.norm, True), (choice.grad, True), (choice.wide_grad, False)):
        for even in (True, False):
            reached = {kernel(of, cols, any_lanes) for _, cols in NORMS if (cols % 8 == 0) == even}
            assert reached == kernels(of, any_lanes)
    for of, groups, any_lanes in ((choice.grad, choice.grad_groups, True),
                                  (choice.wide_grad, choice.wide_grad_groups, False)):
        for rows, cols in MANY_ROWS:
            lanes = of(cols) // 4
            threads = 256 if lanes <= 64 else lanes
            assert rows > 2 * groups(rows, cols) * (threads // lanes)
        assert {kernel(of, cols, any_lanes) for _, cols in MANY_ROWS} == kernels(of, any_lanes) - {(0, 0)}


def test_norm_launches_are_of_a_launchs_size(choice):
    for rows in (1, 2, 3, 4, 2_047, 2_048, 10_000, 1 << 20, (1 << 31) - 1):
        for threads in (128, 192, 256, 512, 1_024):
            n = choice.groups(rows, threads)
            assert 1 <= n <= rows and n * threads < 1 << 32
        for cols in (1, 100, 1_000, 2_000, 4_000, 8_000):
            assert 1 <= choice.grad_groups(rows, cols) <= min(rows, 1_024)
            assert 1 <= choice.wide_grad_groups(rows, cols) <= min(rows, 2_048)
        for cols in (9_000, 20_000, 1 << 24):
            assert 1 <= choice.strips(rows, cols) <= min(rows, 2_048)


def test_norm_gradients_have_no_more_workgroups_than_the_chip_has_room_for(choice):
    """At any number of lanes: 1,024 threads a unit at most, none without a row; and no more partial results
    than the workspace's documented bound, whatever the stream's type."""
    for cols in list(range(1, 600)) + list(range(600, 8_193, 61)) + [1_032, 1_536, 2_048, 4_096, 8_192]:
        for of, groups in ((choice.grad, choice.grad_groups), (choice.wide_grad, choice.wide_grad_groups)):
            lanes = of(cols) // 4
            threads = 256 if lanes <= 64 else lanes
            for rows in (1, 2, 17, 999, 5_000, 131_072, (1 << 31) - 1):
                n = groups(rows, cols)
                assert 1 <= n <= min(-(-rows // (threads // lanes)), 256 * (1_024 // threads), 2_048)
