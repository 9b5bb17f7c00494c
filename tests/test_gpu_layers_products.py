"""Every kernel of the 8-bit product, at sizes that the choice takes it for, against the product in 64 bits
(whole numbers below 2^53: exact). All of the output is compared."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import layers_oracle as O
import paper_2609_22441_amd as P
from gpu_common import note
from layers_common import DEV, F32, HALF_ULP, TINY, TYPES, Output
from layers_sizes import PRODUCTS, SKINNY_LINEAR

pytestmark = pytest.mark.gpu


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def eight_bits(g, rows, k, pad=0):
    """int8 values over the whole range, as a view into rows of `pad` more, with factors of about 1/127."""
    wide = torch.full((rows, k + pad), 77, dtype=torch.int8, device=DEV)
    wide[:, :k] = torch.randint(-128, 128, (rows, k), generator=g, device=DEV).to(torch.int8)
    return wide[:, :k], (torch.rand(rows, generator=g, device=DEV) + 0.5) / 127


def whole(a, b):
    return a.double() @ b.double().t()


def check(o, want, size, out, what):
    """4 * 2^-24 of the terms' magnitude (the sum's conversion, two products, one addition), + half a unit of
    the output's type. NaN where, and only where, NaN is wanted."""
    torch.cuda.synchronize()
    got = o.t.double()
    o.t.fill_(o.fill)
    assert bool((o.wide == o.fill).all()), f"{what}: written outside the output"
    ops = 4 * F32 * size
    near = (got - want).abs() <= ops + HALF_ULP[out] * (want.abs() + ops) + TINY[out]
    bad = ~(near | (got.isnan() & want.isnan()))
    if bool(bad.any()):
        i = tuple(bad.nonzero()[0].tolist())
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} differ, first at {i}: "
                             f"{float(got[i])!r} against {float(want[i])!r}")


@pytest.mark.parametrize("m,n,k,kernel", PRODUCTS)
def test_product(m, n, k, kernel):
    g = gen(m + n + k)
    a, sa = eight_bits(g, m, k, 16 * (m % 2))
    b, sb = eight_bits(g, n, k, 16 * (n % 2))
    sa /= np.sqrt(k)
    bias = torch.randn(n, generator=g, device=DEV) * 10
    s = whole(a, b)
    y = s * sa.double()[:, None] * sb.double()
    for out, with_bias, relu, pad, shift in (("bf16", True, True, 0, 0), ("bf16", False, False, 3, 1),
                                             ("f16", True, False, 8, 8), ("f32", False, True, 3, 1),
                                             ("f32", True, False, 0, 0)):
        what = f"product kernel {kernel} {m}x{n}x{k} {out} bias={with_bias} relu={relu} pad={pad}"
        note(what)
        want = y + bias.double() if with_bias else y
        size = y.abs() + bias.double().abs() if with_bias else y.abs()
        o = Output(m, n, TYPES[out], pad, shift)
        P.cc_matmul_i8(a, sa, b, sb, o.t, bias=bias if with_bias else None, relu=relu)
        check(o, want.clamp(min=0) if relu else want, size, out, what)


@pytest.mark.parametrize("m,n,k,kernel", PRODUCTS)
def test_sums_are_exact_and_rows_alone_give_the_same_bits(m, n, k, kernel):
    """Factors of one: the sum's conversion to 32 bits is the only rounding. With factors and a bias, a few of
    the rows, which another kernel multiplies, have the bits that they have among all."""
    note(f"product bits, kernel {kernel} {m}x{n}x{k}")
    g = gen(m * n)
    (a, sa), (b, sb) = eight_bits(g, m, k), eight_bits(g, n, k)
    a[m // 2], b[n // 2] = -128, -128                          # the largest sum
    out = torch.full((m, n), -7.5, device=DEV)
    P.cc_matmul_i8(a, torch.ones_like(sa), b, torch.ones_like(sb), out)
    torch.cuda.synchronize()
    assert torch.equal(out, whole(a, b).float())
    bias = torch.randn(n, generator=g, device=DEV)
    P.cc_matmul_i8(a, sa, b, sb, out, bias=bias)
    some = torch.tensor([0, m // 3, m // 2, m - 1], device=DEV)
    few = torch.empty(4, n, device=DEV)
    P.cc_matmul_i8(a[some], sa[some], b, sb, few, bias=bias)
    torch.cuda.synchronize()
    assert torch.equal(out[some], few)


def run_linear(m, n, k, dtype, what):
    """Against the oracle's quantisation, and the bits of the two calls that it is made of. A row with an
    infinity is NaN."""
    note(what)
    g = gen(m + 3 * n + k)
    x = torch.randn(m, k + 3, generator=g, device=DEV).to(TYPES[dtype])[:, 1:k + 1]     # aligned to an element
    if m > 3:
        x[3, k // 2] = float("inf")
    padded = -(-k // 16) * 16
    w, sw = eight_bits(g, n, padded)
    w[:, k:] = 0
    sw /= np.sqrt(k)
    bias = torch.randn(n, generator=g, device=DEV)
    ws = torch.full((P.cc_linear_i8_workspace_bytes(m, n, k),), 0xA5, dtype=torch.uint8, device=DEV)
    q, sq = (torch.from_numpy(v).to(DEV) for v in O.quantize(x.float().cpu().numpy()))
    y = whole(q, w) * sq.double()[:, None] * sw.double()
    o = Output(m, n, TYPES[dtype], 3, 1)
    P.cc_linear_i8(x, w, sw, o.t, bias=bias, relu=True, workspace=ws)
    two = torch.empty(m, n, dtype=TYPES[dtype], device=DEV)
    P.cc_quantize_rows(x, q, sq)
    P.cc_matmul_i8(q, sq, w, sw, two, bias=bias, relu=True)
    torch.cuda.synchronize()
    same = (o.t == two) | (o.t.isnan() & two.isnan())
    assert bool(same.all()), what
    want = y + bias.double()
    check(o, torch.where(want.isnan(), want, want.clamp(min=0)), y.abs() + bias.double().abs(), dtype, what)


@pytest.mark.parametrize("m,n,k,kernel", PRODUCTS)
def test_linear(m, n, k, kernel):
    dtype = ("bf16", "f16", "f32")[(m + kernel) % 3]
    run_linear(m, n, k - (n % 2) * 3, dtype, f"linear, product kernel {kernel} {m}x{n}x{k} {dtype}")


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("m,n,k", SKINNY_LINEAR)
def test_linear_of_few_rows(m, n, k, dtype):
    run_linear(m, n, k, dtype, f"linear of few rows {m}x{n}x{k} {dtype}")
