"""The embedding gradient of many tokens (sorted pairs, sums by chunk, fold, join) against 64 bits."""
from __future__ import annotations

import numpy as np
import pytest

from gpu_common import note
from layers_common import rng
from layers_grad import check, rows_on_gpu

pytestmark = pytest.mark.gpu


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
