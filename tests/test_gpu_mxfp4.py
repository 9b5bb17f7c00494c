"""Rows in microscaled 4-bit floating point: every code and scale against the definition, values back, and
products against the 64-bit product of the values that the codes stand for."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import block_oracle as O
import paper_2609_22441_amd as P
from gpu_common import note
from layers_common import DEV, HALF_ULP, TINY, TYPES, Output, assert_close, on_gpu, rng

pytestmark = pytest.mark.gpu


def room(rows, cols, pad=0):
    """(values, scales) of rows in 4 bits, within rows of 16 * pad more bytes."""
    q = torch.full((rows, -(-cols // 128) * 64 + 16 * pad), 0x77, dtype=torch.uint8, device=DEV)
    s = torch.full((rows, -(-cols // 512) * 16 + 16 * pad), 0x77, dtype=torch.uint8, device=DEV)
    return q[:, :q.shape[1] - 16 * pad], s[:, :s.shape[1] - 16 * pad], q, s


def rows_of(r, rows, cols, dtype, wild=True):
    """Rows of every size that the type has, ties and midpoints among them."""
    x = r.standard_normal((rows, cols))
    if wild:
        low, high = {"f32": (-140, 120), "bf16": (-130, 120), "f16": (-22, 13)}[dtype]
        x *= 2.0 ** r.integers(low, high, (rows, -(-cols // 32))).repeat(32, axis=1)[:, :cols]
        tie = r.random(x.shape) < 0.3
        unit = 2.0 ** np.floor(np.log2(np.abs(x) + 1e-300))
        x = np.where(tie, np.round(x / unit * 8) / 8 * unit, x)
    return torch.from_numpy(x).to(TYPES[dtype])


def check_quantize(t, dtype, pad=0, shift=0, out="f32"):
    rows, cols = t.shape
    q, s, q_all, s_all = room(rows, cols, pad)
    P.cc_quantize_mxfp4(on_gpu(t, pad, shift), q, s)
    codes, scales = O.quantize(t.double().numpy())
    assert np.array_equal(s.cpu().numpy(), scales), "scales"
    assert np.array_equal(q.cpu().numpy(), O.packed(codes)), "values"
    if pad:
        assert bool((q_all[:, q.shape[1]:] == 0x77).all()) and bool((s_all[:, s.shape[1]:] == 0x77).all())
    o = Output(rows, cols, TYPES[out], pad, shift)
    P.cc_dequantize_mxfp4(q, s, o.t)
    want = O.values(codes, scales)[:, :cols]
    want = torch.from_numpy(want).to(TYPES[out]).double().numpy()       # one rounding, or none
    assert_close(o.get(), want, 0.0, "back")


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 7), (2, 31), (5, 32), (4, 33), (7, 96), (3, 128),
                                       (2, 129), (5, 500), (3, 512), (2, 513), (3, 1_030), (1, 5_000)])
def test_rows(dtype, rows, cols):
    note(f"mxfp4 rows {rows}x{cols} {dtype}")
    r = rng(rows * 7 + cols)
    for pad, shift, out in ((0, 0, dtype), (8, 8, "f32"), (3, 1, dtype), (1, 0, "bf16")):
        check_quantize(rows_of(r, rows, cols, dtype), dtype, pad, shift, out)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_rows(dtype):
    """Several blocks a thread, the last tile partly filled."""
    note(f"mxfp4 many rows {dtype}")
    r = rng(3)
    for rows, cols in ((1_100, 4_100), (40_000, 130)):
        x = torch.from_numpy(r.standard_normal((rows, cols)).astype(np.float32)).to(TYPES[dtype])
        q, s, _, _ = room(rows, cols)
        P.cc_quantize_mxfp4(x.to(DEV), q, s)
        some = np.unique(np.r_[0, 1, rows - 2, rows - 1, r.integers(0, rows, 12)])
        codes, scales = O.quantize(x[some].double().numpy())
        at = torch.from_numpy(some).to(DEV)
        assert np.array_equal(s[at].cpu().numpy(), scales)
        assert np.array_equal(q[at].cpu().numpy(), O.packed(codes))
        # All of them: the same rows in calls of their own, which take a block a thread.
        for i in range(0, rows, 400):
            q2, s2, _, _ = room(min(400, rows - i), cols)
            P.cc_quantize_mxfp4(x[i:i + 400].to(DEV), q2, s2)
            assert torch.equal(q[i:i + 400], q2) and torch.equal(s[i:i + 400], s2)
        out = torch.empty(rows, cols, dtype=TYPES[dtype], device=DEV)
        P.cc_dequantize_mxfp4(q, s, out)
        assert np.array_equal(out[at].double().cpu().numpy(), O.values(codes, scales)[:, :cols])


def test_ends_of_the_range():
    """Zeros of both signs, subnormal and largest numbers, every midpoint of the grid and its neighbours,
    a block's largest at the border between two scales."""
    note("mxfp4 ends")
    rows = []
    for e in (-149, -148, -130, -127, -126, -125, -124, -20, 0, 60, 120, 125):
        unit = np.float32(2.0 ** e)
        around = []
        for m in np.r_[O.MIDDLE, O.GRID, 7, 1.75]:
            v = np.float32(m * np.float64(unit))
            around += [v, np.nextafter(v, np.float32(0)), np.nextafter(v, np.float32(np.inf))]
        around = [v for v in around if np.isfinite(v)]
        for largest in (4.0, 3.5, np.nextafter(np.float32(3.5), np.float32(0)), 6.9999995, 7.0, 6.0):
            top = np.float32(np.float64(largest) * np.float64(unit))
            if not np.isfinite(top):
                continue
            small = [v for v in around if v <= top]
            for i in range(0, len(small), 31):
                part = small[i:i + 31]
                row = np.zeros(32, dtype=np.float32)
                row[:len(part)] = part
                row[1::2] *= -1
                row[31] = top
                rows.append(row)
    rows += [np.full(32, -0.0, dtype=np.float32), np.full(32, np.finfo(np.float32).max),
             np.full(32, -np.finfo(np.float32).max)]
    t = torch.from_numpy(np.stack(rows).astype(np.float32))
    check_quantize(t, "f32")
    # 6 * 2^126 is 2^128.6: back it is an infinity.
    q, s, _, _ = room(1, 32)
    P.cc_quantize_mxfp4(t[-2:-1].to(DEV), q, s)
    assert int(s[0, 0]) == 253 and int(q[0, 0]) == 0x66


def test_nan_and_infinity_stay_in_their_block():
    note("mxfp4 nan")
    for dtype in ("bf16", "f16", "f32"):
        t = rows_of(rng(1), 4, 100, dtype, wild=False)
        t[1, 40], t[2, 99], t[3, 0] = float("nan"), float("inf"), float("-inf")
        check_quantize(t, dtype, out=dtype)


def quantized(r, rows, k):
    """Rows in 4 bits with scales of many sizes, and their values."""
    codes = r.integers(0, 16, (rows, -(-k // 128) * 128)).astype(np.uint8)
    codes[:, k:] = 0
    scales = np.zeros((rows, -(-k // 512) * 16), dtype=np.uint8)
    blocks = -(-k // 32)
    scales[:, :blocks] = r.integers(115, 132, (rows, blocks))
    return codes, scales, O.values(codes, scales), \
        torch.from_numpy(O.packed(codes)).to(DEV), torch.from_numpy(scales).to(DEV)


def padded(t, pad):
    wide = torch.full((t.shape[0], t.shape[1] + 16 * pad), 0x77, dtype=torch.uint8, device=DEV)
    wide[:, :t.shape[1]] = t
    return wide[:, :t.shape[1]]


def check_product(m, n, k, out="f32", bias=True, relu=False, pad=0, shift=0, seed=0):
    r = rng(m * 31 + n * 7 + k + seed)
    _, _, a, qa, sa = quantized(r, m, k)
    _, _, b, qb, sb = quantized(r, n, k)
    v = r.standard_normal(n).astype(np.float32) * 8 if bias else None
    o = Output(m, n, TYPES[out], pad, shift)
    P.cc_matmul_mxfp4(padded(qa, pad), padded(sa, pad), padded(qb, pad), padded(sb, pad), o.t,
                      bias=None if v is None else torch.from_numpy(v).to(DEV), relu=relu)
    want, e = O.product(a, b, v, relu)
    got = o.get()
    if out == "f16":
        # 65,504 is its largest number and 65,520 half a step beyond: what may lie there rounds to an
        # infinity of its sign.
        over = (np.abs(want) + e >= 65_520) & (got == np.sign(want) * np.inf)
        want = np.where(over, got, want)
    assert_close(got, want, e + HALF_ULP[out] * (np.abs(want) + e) + TINY[out],
                 f"{m}x{n}x{k} {out}")


@pytest.mark.parametrize("m,n,k", [
    (1, 1, 128), (1, 1, 1), (3, 5, 640), (16, 16, 512), (17, 15, 128), (1, 33, 4_096), (16, 100, 5_000),
    (33, 70, 1_152), (64, 64, 256), (65, 129, 384), (128, 64, 2_048), (200, 300, 128),
    (130, 257, 1_030), (256, 256, 512), (300, 520, 2_176), (1, 4_100, 96), (500, 20, 3_000)])
def test_product(m, n, k):
    note(f"mxfp4 product {m}x{n}x{k}")
    check_product(m, n, k)
    check_product(m, n, k, "bf16", relu=True, pad=1, shift=1, seed=1)
    check_product(m, n, k, "f16", bias=False, pad=3, seed=2)


def test_product_of_nothing():
    note("mxfp4 product of nothing")
    out = torch.full((3, 5), 7.0, device=DEV)
    bias = torch.arange(5.0, device=DEV) - 2
    none = [torch.empty(rows, 0, dtype=torch.uint8, device=DEV) for rows in (3, 5)]
    P.cc_matmul_mxfp4(none[0], none[0], none[1], none[1], out, bias=bias, relu=True)
    assert torch.equal(out, bias.clamp(min=0).expand(3, 5))
    q, s, _, _ = room(0, 128)
    w, sw, _, _ = room(5, 128)
    P.cc_matmul_mxfp4(q, s, w, sw, torch.empty(0, 5, device=DEV))
    P.cc_quantize_mxfp4(torch.empty(0, 128, device=DEV), q, s)
    P.cc_dequantize_mxfp4(q, s, torch.empty(0, 128, device=DEV))


@pytest.mark.parametrize("m,n,k", [(4, 40, 96), (300, 300, 640)])
def test_what_lies_behind_k_has_no_part(m, n, k):
    """Scales behind k's blocks may hold anything (NaN here), and an infinite scale gives NaN where it is
    part of the sum, and only there."""
    note(f"mxfp4 behind k {m}x{n}x{k}")
    r = rng(k)
    _, scales, a, qa, sa = quantized(r, m, k)
    _, _, b, qb, sb = quantized(r, n, k)
    used = -(-k // 128) * 4
    sa[:, used:] = 255
    sb[:, used:] = 255
    sa[1, 0] = 255
    sb[2, 1] = 255
    out = torch.empty(m, n, device=DEV)
    P.cc_matmul_mxfp4(qa, sa, qb, sb, out)
    want, e = O.product(a, b)
    want[1], want[:, 2] = np.nan, np.nan
    assert_close(out.double().cpu().numpy(), want, e, "behind k")


@pytest.mark.parametrize("m,n,k", [(1, 64, 96), (1, 512, 4_096), (5, 70, 130), (16, 64, 1_000),
                                   (17, 64, 1_000), (200, 256, 96), (300, 300, 700), (40, 33, 7)])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_linear(dtype, m, n, k):
    """The linear layer is quantisation and product, bit by bit where both take the same kernel, within
    the bounds of the 64-bit product anyway."""
    note(f"mxfp4 linear {m}x{n}x{k} {dtype}")
    r = rng(m + n + k)
    x, w = rows_of(r, m, k, dtype, wild=False), rows_of(r, n, k, "f32", wild=False)
    qw, sw, _, _ = room(n, k)
    P.cc_quantize_mxfp4(w.to(DEV), qw, sw)
    bias = torch.from_numpy(r.standard_normal(n)).float()
    ws = torch.full((P.cc_linear_mxfp4_workspace_bytes(m, n, k) + 32,), 0x55, dtype=torch.uint8,
                    device=DEV)
    for pad, shift in ((0, 0), (3, 1)):
        o = Output(m, n, TYPES[dtype], pad, shift)
        P.cc_linear_mxfp4(on_gpu(x, pad, shift), qw, sw, o.t, bias=bias.to(DEV), relu=True,
                          workspace=ws[:-32])
        a = O.values(*O.quantize(x.double().numpy()))
        b = O.values(*O.quantize(w.double().numpy()))
        want, e = O.product(a, b, bias.double().numpy(), True)
        assert_close(o.get(), want, e + HALF_ULP[dtype] * (np.abs(want) + e) + TINY[dtype], "linear")
    assert bool((ws[-32:] == 0x55).all())
