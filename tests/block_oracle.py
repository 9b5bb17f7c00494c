"""The block norms, their gradient and microscaled 4-bit rows in 64 bits with NumPy, from the formulas in
include/cc_layers.h. The norms come with bounds: every value carries how far a computation in 32 bits
may be from it, by the rounding of each of its operations (2^-24 relative) and what its operands
carry."""
from __future__ import annotations

import numpy as np

from layers_common import F32

NONE, RMS, LAYER = 0, 1, 2
LINEAR, SIGMOID = 0, 1


class Bound:
    """A value in 64 bits and the largest error of its computation in 32."""

    def __init__(self, v, e=0.0):
        self.v = np.asarray(v, dtype=np.float64)
        self.e = np.broadcast_to(np.asarray(e, dtype=np.float64), self.v.shape)

    @staticmethod
    def of(x):
        return x if isinstance(x, Bound) else Bound(x)

    def __add__(self, o):
        o = Bound.of(o)
        v = self.v + o.v
        return Bound(v, (self.e + o.e) * (1 + F32) + F32 * np.abs(v))

    __radd__ = __add__

    def __neg__(self):
        return Bound(-self.v, self.e)

    def __sub__(self, o):
        return self + (-Bound.of(o))

    def __mul__(self, o):
        o = Bound.of(o)
        v = self.v * o.v
        e = np.abs(self.v) * o.e + np.abs(o.v) * self.e + self.e * o.e
        return Bound(v, e * (1 + F32) + F32 * np.abs(v))

    __rmul__ = __mul__

    def sum(self, axis, roundings):
        """A sum whose terms pass at most `roundings` additions each."""
        v = self.v.sum(axis, keepdims=True)
        size = (np.abs(self.v) + self.e).sum(axis, keepdims=True)
        return Bound(v, self.e.sum(axis, keepdims=True) + roundings * F32 * size)


def mean_of(s, cols):
    """A sum times 1 / cols: the factor's rounding and the product's."""
    return Bound(s.v / cols, s.e / cols + 2 * F32 * (np.abs(s.v) + s.e) / cols)


def inverse_size(sum_, cols, eps):
    """1 / sqrt(sum / cols + eps): the root halves its operand's relative error, and is itself within a unit
    in the last place."""
    q = mean_of(sum_, cols) + np.float64(np.float32(eps))
    v = q.v ** -0.5
    low = np.maximum(q.v - q.e, q.v * 0.25)
    return Bound(v, v * (0.5 * q.e / low * (q.v / low) ** 0.5 + 2 * F32))


def unit(v, norm, eps):
    """(v normalised, 1 / its size). A term of a row's sum passes the additions of its lane (one in 256
    columns, or 16), those between 64 lanes and those between 16 wavefronts."""
    cols = v.v.shape[1]
    roundings = 40 + cols // 256
    if norm == NONE:
        return v, Bound(1.0)
    if norm == LAYER:
        s = v.sum(1, roundings)
        v = v - mean_of(s, cols)
    r = inverse_size((v * v).sum(1, roundings), cols, eps)
    return v * r, r


def mean(v):
    cols = v.v.shape[1]
    return mean_of(v.sum(1, 40 + cols // 256), cols)


def gate_of(u, kind):
    """(g, its derivative). exp(-|u|) by 2^x: the product with log2 e is off by 2 units of |u|, the
    power by one of its last place; a reciprocal by one; below 2^-126 nothing is left."""
    if u is None:
        return Bound(1.0), Bound(1.0)
    if kind == LINEAR:
        return Bound(u), Bound(1.0)
    e = np.exp(-np.abs(u))
    e = Bound(e, e * (2 * np.abs(u) + 3) * F32 + 2.0 ** -126)
    one = 1 + e
    r = 1 / one.v
    r = Bound(r, r * (one.e / (one.v - one.e) + 2 * F32))
    g = e * r
    return Bound(np.where(u < 0, g.v, r.v), np.where(u < 0, g.e, r.e)), e * r * r


def forward(c):
    """fn, its factor, n, g, slope, y, yn and its factor of a call described by the dict c."""
    f = Bound(c["f"])
    fn, r = unit(f, c["post_norm"], c["post_eps"])
    n = fn
    if c.get("post_weight") is not None:
        n = n * c["post_weight"]
    if c.get("post_bias") is not None:
        n = n + c["post_bias"]
    g, slope = gate_of(c.get("gate"), c["gate_kind"])
    scale = np.float64(np.float32(c["scale"]))
    y = scale * g * n
    if c.get("x") is not None:
        y = y + c["x"]
    yn, ry = unit(y, c["pre_norm"], c["pre_eps"])
    return fn, r, n, g, slope, y, yn, ry


def norm(c):
    """(y, h) as Bounds."""
    *_, y, yn, _ = forward(c)
    h = yn
    if c.get("pre_weight") is not None:
        h = h * c["pre_weight"]
    if c.get("pre_bias") is not None:
        h = h + c["pre_bias"]
    return y, h


def back(t, vn, r, kind):
    if kind == NONE:
        return t
    d = t - vn * mean(t * vn)
    if kind == LAYER:
        d = d - mean(t)
    return d * r


def norm_grad(c, dy, dh):
    """dx, df, dgate and the four vectors' gradients as Bounds; None where there is none."""
    fn, r, n, g, slope, _, yn, ry = forward(c)
    rows = fn.v.shape[0]
    through = min(rows, 64 + rows // 16)          # additions that a row's term passes
    out = dict(d_pre_weight=None, d_pre_bias=None, dgate=None)
    d = Bound(np.zeros_like(fn.v) if dy is None else dy)
    if dh is not None:
        dh = Bound(dh)
        t = dh if c.get("pre_weight") is None else dh * c["pre_weight"]
        d = d + back(t, yn, ry, c["pre_norm"])
        out["d_pre_weight"] = (dh * yn).sum(0, through)
        out["d_pre_bias"] = dh.sum(0, through)
    out["dx"] = d
    d = d * np.float64(np.float32(c["scale"]))
    if c.get("gate") is not None:
        out["dgate"] = d * n * slope
    dg = d * g
    out["d_post_weight"] = (dg * fn).sum(0, through)
    out["d_post_bias"] = dg.sum(0, through)
    w = dg if c.get("post_weight") is None else dg * c["post_weight"]
    out["df"] = back(w, fn, r, c["post_norm"])
    return out


# ---- microscaled 4-bit floating point ----

GRID = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
MIDDLE = (GRID[1:] + GRID[:-1]) / 2


def exponent(most):
    """s of a block's largest magnitude (finite), by comparison: the least e with the magnitude below
    1.75 * 2^(e - 127), less 2."""
    if most == 0:
        return 0
    e = int(np.floor(np.log2(most))) + 127 - 1
    while most >= 1.75 * 2.0 ** (e - 127):
        e += 1
    return max(e - 2, 0)


def quantize(x):
    """(codes [rows, padded to 128], s [rows, padded to 16 of 32 columns])."""
    rows, cols = x.shape
    codes = np.zeros((rows, -(-cols // 128) * 128), dtype=np.uint8)
    scales = np.zeros((rows, -(-cols // 512) * 16), dtype=np.uint8)
    for r in range(rows):
        for b in range(-(-cols // 32)):
            v = x[r, b * 32:(b + 1) * 32]
            if not np.isfinite(v).all():
                scales[r, b] = 255
                continue
            s = exponent(np.abs(v).max())
            scales[r, b] = s
            a = np.abs(v) / 2.0 ** (s - 127)
            above = (a[:, None] > MIDDLE).sum(1)
            tie = (a[:, None] == MIDDLE).any(1)
            code = above + (tie & (above % 2 == 1))
            codes[r, b * 32:b * 32 + v.size] = code | np.signbit(v).astype(np.uint8) << 3
    return codes, scales


def packed(codes):
    return codes[:, 0::2] | codes[:, 1::2] << 4


def values(codes, scales):
    """In 64 bits; NaN where s is 255."""
    v = np.where(codes & 8, -1.0, 1.0) * GRID[codes & 7]
    unit_ = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return v * np.repeat(unit_, 32, axis=1)[:, :codes.shape[1]]


def product(a, b, bias=None, relu=False):
    """(result, bound) of values [m, k] and [n, k]. Products are exact. An instruction adds 64 or 128 of
    them to the sum so far, whatever its way of rounding within a unit in the last place of the
    sum of magnitudes; the sums of up to 8 wavefronts meet, and the bias is added."""
    with np.errstate(invalid="ignore"):
        v, size = a @ b.T, np.abs(a) @ np.abs(b).T
        steps = -(-a.shape[1] // 64) + 10
        e = steps * 2 * F32 * size
        if bias is not None:
            v = v + bias
        e = e + F32 * np.abs(v)
        return (np.maximum(v, 0) if relu else v), e
