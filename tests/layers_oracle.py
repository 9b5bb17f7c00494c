"""Plain numpy forms of the scoring model's input layer, in 64 bits, one step of the definition at a
time; the tests compare the kernels with these. No code is shared with the library."""
from __future__ import annotations

import numpy as np

M32 = (1 << 32) - 1


def philox(counter, key):
    """Philox4x32-10 (Salmon et al., SC 2011): the four words of one counter, in Python integers."""
    c, k = list(counter), list(key)
    for _ in range(10):
        a, b = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
        c = [(b >> 32) ^ c[1] ^ k[0], b & M32, (a >> 32) ^ c[3] ^ k[1], a & M32]
        k = [(k[0] + 0x9E3779B9) & M32, (k[1] + 0xBB67AE85) & M32]
    return c


def threshold(p):
    return 65536 - int(np.floor(65536 * p + 0.5))


def kept(rows, cols, p, seed, site=0, first_row=0):
    """Dropout's mask, [rows, cols] of bool: philox for all counters at once."""
    blocks = (cols + 7) // 8
    u = np.uint64
    row = np.array([first_row + r for r in range(rows)], dtype=u)[:, None] + np.zeros(blocks, u)
    c = [row & u(M32), row >> u(32), np.arange(blocks, dtype=u)[None, :] + np.zeros((rows, 1), u),
         np.full((rows, blocks), site, u)]
    k = [seed & M32, seed >> 32]
    for _ in range(10):
        a, b = c[0] * u(0xD2511F53), c[2] * u(0xCD9E8D57)
        c = [(b >> u(32)) ^ c[1] ^ u(k[0]), b & u(M32), (a >> u(32)) ^ c[3] ^ u(k[1]), a & u(M32)]
        k = [(k[0] + 0x9E3779B9) & M32, (k[1] + 0xBB67AE85) & M32]
    out = np.empty((rows, blocks, 8), dtype=bool)
    for i in range(8):
        out[:, :, i] = ((c[i // 2] >> u(16 * (i % 2))) & u(0xFFFF)) < u(threshold(p))
    return out.reshape(rows, blocks * 8)[:, :cols]


def mask_or_all(rows, cols, drop):
    """The mask of drop = dict(p, seed, site, first_row), and the factor of what is kept."""
    if not drop or drop["p"] == 0:
        return np.ones((rows, cols), bool), 1.0
    t = threshold(drop["p"])
    return kept(rows, cols, **drop), 65536 / t if t else 0.0


def lookup(table, ids, scale=1.0, drop=None):
    """float64 [n, cols] of a float64 table."""
    n, cols = len(ids), table.shape[1]
    keep, factor = mask_or_all(n, cols, drop)
    out = np.zeros((n, cols))
    for t, i in enumerate(ids):
        if 0 <= i < len(table):
            out[t] = np.where(keep[t], table[i], 0.0) * (scale * factor)
    return out


def grad(ids, dout, rows, scale=1.0, drop=None):
    """(gradient, sum of the magnitudes that were added, additions) of float64 dout."""
    n, cols = dout.shape
    keep, factor = mask_or_all(n, cols, drop)
    g, size = np.zeros((rows, cols)), np.zeros((rows, cols))
    count = np.zeros((rows, 1))
    for t, i in enumerate(ids):
        if 0 <= i < rows:
            d = np.where(keep[t], dout[t], 0.0) * (scale * factor)
            g[i] += d
            size[i] += np.abs(d)
            count[i] += 1
    return g, size, count


def dropout(x, drop, residual=None):
    keep, factor = mask_or_all(*x.shape, drop)
    y = np.where(keep, x, 0.0) * factor
    return y if residual is None else y + residual


def quantize(x):
    """(q, scales) of float32 rows, each step rounded to 32 bits as the definition says."""
    x = x.astype(np.float32)
    n, cols = x.shape
    q = np.zeros((n, (cols + 15) // 16 * 16), np.int8)
    scales = np.zeros(n, np.float32)
    for r in range(n):
        most = np.max(np.abs(x[r]))
        if not np.isfinite(x[r]).all():
            scales[r] = np.nan
        elif most > 0:
            # rows below 2^-60 are raised by 2^64 first, which changes no digit of the quotient
            up = np.float32(2.0 ** 64) if most < 2.0 ** -60 else np.float32(1)
            scales[r] = most / np.float32(127)
            q[r, :cols] = np.rint((x[r] * up) * (np.float32(127) / (most * up))).astype(np.int8)
    return q, scales


def product(a, a_scales, b, b_scales, bias=None, relu=False):
    """(float64 result, magnitude of its two terms)."""
    s = a.astype(np.int64) @ b.astype(np.int64).T
    y = s * a_scales.astype(np.float64)[:, None] * b_scales.astype(np.float64)
    size = np.abs(y)
    if bias is not None:
        y = y + bias.astype(np.float64)
        size = size + np.abs(bias.astype(np.float64))
    return (np.maximum(y, 0) if relu else y), size
