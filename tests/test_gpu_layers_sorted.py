"""Every form of the embedding gradient (one launch; windows; sorted pairs with sums by chunk, fold and join)
against 64 bits, in each type, with and without dropout, aligned or not."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import layers_oracle as O
from gpu_common import note
from layers_common import rng
from layers_grad import check, kept, outside, rows_on_gpu
from layers_sizes import GRAD

pytestmark = pytest.mark.gpu

DROP = dict(p=0.2, seed=0x0FED_CBA9_8765_4321, site=4, first_row=(1 << 32) - 900)
LARGE = 1 << 25                 # elements from which a size runs in fewer combinations
EVEN, ODD = (0, 0), (3, 1)      # elements after a row and before the first one


def test_the_mask_is_the_oracles():
    note("grad: mask on the GPU")
    for rows, cols in ((2_000, 21), (5, 1_000)):
        assert (kept(rows, cols, **DROP).cpu().numpy() == O.kept(rows, cols, **DROP)).all()


def zipf(r, n, rows):
    w = np.arange(1, rows + 1) ** -1.1
    ranks = np.searchsorted(np.cumsum(w / w.sum()), r.random(n)).clip(0, rows - 1)
    return r.permutation(rows)[ranks]


def combinations(n, cols):
    """type of the rows, type of the table, dropout, layout, accumulate"""
    if n * cols > LARGE:
        return [("bf16", "f32", True, EVEN, False), ("bf16", "bf16", False, ODD, True),
                ("f32", "f32", True, ODD, False), ("f16", "f16", True, EVEN, True)]
    return [(dtype, table, drop, layout, drop == (layout == ODD))
            for dtype, table in (("bf16", "f32"), ("f16", "f32"), ("f32", "f32"), ("bf16", "bf16"),
                                 ("f16", "f16"))
            for drop in (False, True) for layout in (EVEN, ODD)]


@pytest.mark.parametrize("n,rows,cols", GRAD)
def test_every_form(n, rows, cols):
    r = rng(n + rows + cols)
    ids = outside(r, zipf(r, n, rows).astype(np.int64 if cols % 2 else np.int32), rows, 0.03)
    for dtype, table, drop, layout, accumulate in combinations(n, cols):
        what = f"{dtype} into {table}, dropout {drop}, layout {layout}, accumulate {accumulate}"
        note(f"grad: n={n} rows={rows} cols={cols} {what}")
        d = rows_on_gpu(n, cols, dtype, n, *layout)
        check(ids, d, rows, table, scale=0.7, drop=DROP if drop else None, accumulate=accumulate,
              pad=layout[0], shift=layout[1], what=what)
        del d
    torch.cuda.empty_cache()


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("n,rows,cols", [(8_192, 9_000, 4_096), (8_192, 300, 4_096),
                                         (70_000, 70_000, 520), (70_000, 3_000, 520)])
def test_ids_outside_the_table_end_anywhere_in_a_chunk(n, rows, cols, accumulate):
    """Chunks of 16 tokens, joined at once or folded first. The valid ids end at each place of a chunk in
    turn, and whole chunks of ids outside the table follow: every row has its sum, and only rows are
    written."""
    note(f"grad: valid ids end in a chunk, n={n} rows={rows} cols={cols} accumulate={accumulate}")
    r = rng(n + rows)
    d = rows_on_gpu(n, cols, "bf16", n)
    for valid in range(n - 200, n - 184):
        note(f"  {valid} valid ids")
        inside = r.permutation(rows)[:valid] if rows >= valid else r.integers(0, rows, valid)
        ids = np.concatenate([inside, r.choice([-1, rows, -(1 << 40), 1 << 40], n - valid)])
        check(r.permutation(ids), d, rows, "f32", accumulate=accumulate, what=f"{valid} valid")
