"""Lookup and dropout of many narrow rows (four blocks of 8 columns to a thread: fewer than 64 blocks to a row,
2^19 blocks and more in all) against 64 bits: rows of the width that the join writes among them, and a table of
51 positions of 3 columns."""
from __future__ import annotations

import pytest
import torch

import layers_oracle as O
import paper_2609_22441_amd as P
from gpu_common import note
from layers_common import DEV, F32, HALF_ULP, TINY, TYPES, Output
from layers_grad import kept, rows_on_gpu

pytestmark = pytest.mark.gpu

DROP = dict(p=0.3, seed=0x1234_5678_9ABC_DEF0, site=5, first_row=(1 << 32) - 1_000)
# Blocks of a row: 12 (32-bit rows exchange pieces by four lanes), 16 (by eight), 9 (not at all), 13, 1, 63.
SIZES = [(50_000, 96), (40_000, 128), (60_000, 72), (44_000, 97), (600_000, 3), (9_000, 504)]
LAYOUTS = [(0, 0), (8, 8), (3, 1)]     # elements after a row, and before the first one


def check(o, want, terms, out, what):
    """One product by a factor that is itself rounded, one addition: 3 * 2^-24 of the terms' magnitude, + half a
    unit of the output's type."""
    torch.cuda.synchronize()
    got = o.t.double()
    o.t.fill_(o.fill)
    assert bool((o.wide == o.fill).all()), f"{what}: written outside the output"
    ops = 3 * F32 * terms
    bad = ~((got - want).abs() <= ops + HALF_ULP[out] * (want.abs() + ops) + TINY[out])
    if bool(bad.any()):
        i = tuple(bad.nonzero()[0].tolist())
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} differ, first at {i}: "
                             f"{float(got[i])!r} against {float(want[i])!r}")


@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_dropout(rows, cols, dtype):
    keep = kept(rows, cols, **DROP)
    for pad, shift in LAYOUTS:
        for residual in (False, True):
            what = f"dropout {rows}x{cols} {dtype} residual={residual} pad={pad}"
            note(what)
            x = rows_on_gpu(rows, cols, dtype, rows, pad, shift)
            want = torch.where(keep, x.double() * 65536 / O.threshold(DROP["p"]), 0.0)
            terms, res = want.abs(), None
            if residual:
                res = rows_on_gpu(rows, cols, dtype, rows + 1, pad, shift)
                want, terms = want + res.double(), terms + res.double().abs()
            o = Output(rows, cols, TYPES[dtype], pad, shift)
            P.cc_dropout(x, o.t, residual=res, **DROP)
            check(o, want, terms, dtype, what)


@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("dtype,out", [("bf16", "bf16"), ("f16", "f16"), ("f32", "f32"), ("f32", "bf16"),
                                       ("f32", "f16")])
def test_lookup(rows, cols, dtype, out):
    keep, n_rows = kept(rows, cols, **DROP), 51
    g = torch.Generator(device=DEV).manual_seed(cols)
    ids = torch.randint(-1, n_rows + 1, (rows,), generator=g, device=DEV)
    found = ((ids >= 0) & (ids < n_rows))[:, None]
    for pad, shift in LAYOUTS:
        table = rows_on_gpu(n_rows, cols, dtype, cols, pad, shift)
        for drop in (False, True):
            what = f"lookup {rows}x{cols} {dtype} -> {out} dropout={drop} pad={pad}"
            note(what)
            factor = 1.7 * 65536 / O.threshold(DROP["p"]) if drop else 1.7
            want = torch.where(found & keep if drop else found,
                               table.double()[ids.clamp(0, n_rows - 1)] * factor, 0.0)
            o = Output(rows, cols, TYPES[out], pad, shift)
            P.cc_embedding_lookup(table, ids.int() if pad else ids, o.t, scale=1.7,
                                  **(DROP if drop else {}))
            check(o, want, want.abs(), out, what)
