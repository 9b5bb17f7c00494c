"""The embedding gradient against its definition in 64 bits, summed on the GPU with torch's index_add_: for
calls too large for numpy, whose launches and chunks smaller ones do not reach."""
from __future__ import annotations

import numpy as np
import torch

import layers_oracle as O
import paper_2609_22441_amd as P
from layers_common import DEV, F32, HALF_ULP, TINY, TYPES, Output


def outside(r, ids, rows, share):
    """A share of the ids replaced by ones outside the table: of either end, and far from it."""
    bad = np.array([-1, rows, np.iinfo(ids.dtype).min, np.iinfo(ids.dtype).max], ids.dtype)
    at = r.permutation(len(ids))[:round(len(ids) * share)]
    ids[at] = bad[r.integers(0, 4, len(at))]
    return ids


def rows_on_gpu(n, cols, dtype, seed, pad=0, shift=0):
    """N(0, 1) rows in GPU memory, a view `shift` elements into rows of `pad` more, NaN around it."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    wide = torch.full((n * (cols + pad) + shift + pad,), float("nan"), dtype=TYPES[dtype], device=DEV)
    view = wide[shift:shift + n * (cols + pad)].view(n, cols + pad)[:, :cols]
    view.copy_(torch.randn(n, cols, generator=g, device=DEV))
    return view


def kept(rows, cols, p, seed, site=0, first_row=0):
    """layers_oracle.kept on the GPU, some rows at a time: products modulo 2^64, whose halves are exact."""
    blocks = (cols + 7) // 8
    keep = torch.empty(rows, blocks, 8, dtype=torch.bool, device=DEV)
    step = max(1, (1 << 22) // blocks)
    for i in range(0, rows, step):
        row = torch.arange(first_row + i, first_row + min(i + step, rows), device=DEV)[:, None]
        c = [row & O.M32, row >> 32, torch.arange(blocks, device=DEV)[None, :],
             torch.full((1, 1), site, device=DEV)]
        k = [seed & O.M32, seed >> 32]
        for _ in range(10):
            a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
            c = [(b >> 32 & O.M32) ^ c[1] ^ k[0], b & O.M32, (a >> 32 & O.M32) ^ c[3] ^ k[1], a & O.M32]
            k = [(k[0] + 0x9E3779B9) & O.M32, (k[1] + 0xBB67AE85) & O.M32]
        for j in range(8):
            keep[i:i + step, :, j] = (c[j // 2] >> (16 * (j % 2)) & 0xFFFF) < O.threshold(p)
    return keep.view(rows, blocks * 8)[:, :cols]


def sums(ids, d, rows, keep, factor):
    """(gradient, sum of the magnitudes that were added, additions) in 64 bits. Tokens go round several tables,
    which are added up at the end: a row that takes most of the tokens is slow as one."""
    n, cols = d.shape
    tables = min(1024, max(1, (1 << 25) // ((rows + 1) * (cols + 1))))
    to = torch.where((ids >= 0) & (ids < rows), ids.long(), rows)           # the last: ids outside
    to = to + torch.arange(n, device=DEV) % tables * (rows + 1)
    want, size = (torch.zeros(tables * (rows + 1), cols, dtype=torch.float64, device=DEV)
                  for _ in range(2))
    step = max(1, (1 << 25) // cols)
    for i in range(0, n, step):
        x = d[i:i + step].double() * factor
        if keep is not None:
            x = torch.where(keep[i:i + step], x, 0.0)
        want.index_add_(0, to[i:i + step], x)
        size.index_add_(0, to[i:i + step], x.abs())
    count = torch.bincount(to, minlength=tables * (rows + 1)).double()[:, None]
    return [t.view(tables, rows + 1, -1).sum(0)[:rows] for t in (want, size, count)]


def check(ids, d, rows, table, scale=1.0, drop=None, accumulate=False, pad=0, shift=0, what=""):
    """One call against the sums above. Tolerance: (additions + 2, and one for the old value) * 2^-24 of the
    sum of magnitudes, + half a unit of the table's type. Rows that no id points at are zeros, or unchanged;
    what lies around the table, two rows after it among them, stays as it is."""
    n, cols = d.shape
    ids = torch.from_numpy(ids).to(DEV)
    keep, factor = None, scale
    if drop:
        keep = kept(n, cols, **drop)
        factor = scale * 65536 / O.threshold(drop["p"])
    want, size, count = sums(ids, d, rows, keep, factor)
    o = Output(rows + 2, cols, TYPES[table], pad, shift)
    g = torch.Generator(device=DEV).manual_seed(rows)
    if accumulate:
        o.t[:rows].copy_(torch.randn(rows, cols, generator=g, device=DEV))
    before = o.t[:rows].double()
    ws = torch.full((P.cc_embedding_grad_workspace_bytes(n, rows, cols),), 0xA5, dtype=torch.uint8,
                    device=DEV)
    P.cc_embedding_grad(ids, d, o.t[:rows], ws, scale=scale, accumulate=accumulate, **(drop or {}))
    torch.cuda.synchronize()
    got = o.t[:rows].double()
    o.t[:rows] = o.fill
    assert bool((o.wide == o.fill).all()), f"{what}: written outside the table"
    touched = (count > 0).expand_as(want)
    rest = before if accumulate else torch.zeros_like(got)
    assert torch.equal(got[~touched], rest[~touched]), f"{what}: rows without ids"
    if accumulate:
        want, size, count = want + before, size + before.abs(), count + 1
    ops = (count + 2) * F32 * size
    bad = touched & ~((got - want).abs() <= ops + HALF_ULP[table] * (want.abs() + ops) + TINY[table])
    if bool(bad.any()):
        r, c = bad.nonzero()[0].tolist()
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} differ, first at {(r, c)}: "
                             f"{float(got[r, c])!r} against {float(want[r, c])!r}")
