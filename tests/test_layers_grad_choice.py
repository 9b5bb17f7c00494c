"""The embedding gradient's choice of form (csrc/grad_choice.h, compiled for the host): the sizes of the GPU
tests reach every form, and the rule's edges."""
from __future__ import annotations

import ctypes
import subprocess
import tempfile
from pathlib import Path

import numpy as np
import pytest

from layers_sizes import GRAD
from paper_2609_22441_amd import layers as Y

CSRC = Path(__file__).resolve().parent.parent / "paper_2609_22441_amd" / "csrc"
SMALL, WINDOWS, SORTED = range(3)

SHIM = """#include "grad_choice.h"
extern "C" void choice(int64_t n, int64_t rows, int32_t cols, int64_t *out) {
    const ccj::GradPlan p = ccj::grad_plan(n, rows, cols);
    out[0] = p.window.count == 1 ? 0 : p.window.count ? 1 : 2;
    out[1] = p.lanes;
    out[2] = p.window.count ? p.window.tokens : p.chunk;
    out[3] = p.folds > 0;
    out[4] = p.sort.passes;
    out[5] = p.bytes;
}
"""


@pytest.fixture(scope="module")
def choice():
    with tempfile.TemporaryDirectory() as d:
        src, out = Path(d) / "choice.cpp", Path(d) / "choice.so"
        src.write_text(SHIM)
        subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-shared", "-fPIC", f"-I{CSRC}",
                        str(src), "-o", str(out)], check=True)
        lib = ctypes.CDLL(str(out))

    def call(n, rows, cols):
        """(form, lanes to a row, tokens of a window or chunk, folded, digit passes, bytes)"""
        r = (ctypes.c_int64 * 6)()
        lib.choice(ctypes.c_int64(n), ctypes.c_int64(rows), ctypes.c_int32(cols), r)
        return tuple(r)
    return call


def kind(c):
    """What tells launches apart: of one launch and of windows the lanes, of sorted pairs the chunks too
    (up to 16, or longer) and the fold."""
    form, lanes, tokens, folded = c[:4]
    return (form, lanes) if form != SORTED else (form, lanes, min(tokens, 32), folded)


def test_the_gpu_tests_reach_every_form(choice):
    reached = {kind(choice(*size)) for size in GRAD}
    r = np.random.default_rng(1)
    for _ in range(100_000):
        n, rows, cols = (int(round(np.exp(r.uniform(0, np.log(most)))))
                         for most in (1 << 24, 1 << 24, 8_192))
        if n * cols <= 1 << 30:
            assert kind(choice(n, rows, cols)) in reached, (n, rows, cols)
    assert {(SORTED, lanes, chunk, 1) for lanes in (4, 16, 64) for chunk in (8, 16, 32)} <= reached
    assert {(SORTED, lanes, 8, 0) for lanes in (4, 16, 64)} | {(SORTED, 64, 16, 0)} <= reached
    assert {(form, lanes) for form in (SMALL, WINDOWS) for lanes in (4, 16, 64)} <= reached
    assert {choice(*size)[4] for size in GRAD if choice(*size)[0] == SORTED} == {1, 2, 3}
    assert {choice(*size)[2] for size in GRAD if choice(*size)[0] == WINDOWS} == {128, 256, 512, 1_024}


@pytest.mark.parametrize("n,rows,cols,want", [
    (4_096, 129, 128, (SMALL, 16)), (4_097, 129, 128, (SORTED, 16, 8, 0)),
    (1_024, 128, 129, (SMALL, 64)), (1_025, 128, 129, (WINDOWS, 64)), (1_025, 129, 129, (SORTED, 64, 8, 0)),
    (16_384, 129, 128, (SORTED, 16, 8, 0)), (16_392, 129, 128, (SORTED, 16, 8, 1)),
    (65_535, 129, 512, (SORTED, 64, 8, 1)), (65_536, 129, 512, (SORTED, 64, 16, 1)),
    (8_192, 129, 4_096, (SORTED, 64, 16, 0)), (8_191, 129, 4_096, (SORTED, 64, 8, 1)),
    (262_143, 129, 128, (SORTED, 16, 8, 1)), (262_144, 129, 128, (SORTED, 16, 16, 1)),
    (524_288, 129, 128, (SORTED, 16, 32, 1)), (2_097_152, 129, 32, (SORTED, 4, 32, 1)),
])
def test_edges(choice, n, rows, cols, want):
    assert kind(choice(n, rows, cols)) == want


def test_the_workspace_is_the_plans(choice):
    for size in GRAD + [(1, 1, 1), (0, 700, 40), ((1 << 31) - 1, (1 << 31) - 2, 8)]:
        assert choice(*size)[5] == Y.cc_embedding_grad_workspace_bytes(*size)
