"""Every kernel of the 4-bit product, at sizes that the choice takes it for, against the product in 64 bits
of the values that the codes stand for. All of the output is compared."""
from __future__ import annotations

import pytest
import torch

import paper_2609_22441_amd as P
from block_sizes import INSIDE, OUTSIDE, PRODUCTS
from gpu_common import note
from layers_common import DEV, F32, HALF_ULP, TINY, TYPES, Output

pytestmark = pytest.mark.gpu

GRID = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, 0, -0.5, -1, -1.5, -2, -3, -4, -6], dtype=torch.float64)


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def four_bits(g, rows, k, pad=0):
    """Rows in 4 bits within rows of `pad` more bytes, scales from 2^-8 to 2^3, NaN where no block is;
    and their values."""
    width, scale_width, blocks = -(-k // 128) * 64, -(-k // 512) * 16, -(-k // 128) * 4
    q = torch.randint(0, 256, (rows, width + pad), generator=g, device=DEV).to(torch.uint8)
    s = torch.full((rows, scale_width + pad), 255, dtype=torch.uint8, device=DEV)
    s[:, :blocks] = torch.randint(119, 131, (rows, blocks), generator=g, device=DEV).to(torch.uint8)
    q, s = q[:, :width], s[:, :scale_width]
    return q, s, values(q, s)


def values(q, s):
    codes = torch.stack([q & 15, q >> 4], 2).view(q.shape[0], -1).long()
    unit = torch.pow(2.0, s[:, :q.shape[1] // 16].double() - 127)
    return GRID.to(DEV)[codes] * unit.repeat_interleave(32, dim=1)


def check(o, want, size, steps, out, what):
    """A unit in the last place of the sum of magnitudes for each of `steps` matrix instructions (of 64 or
    more of k) and of up to 8 sums that meet, half of one for the bias, half a unit of the output's
    type."""
    torch.cuda.synchronize()
    got = o.t.double()
    o.t.fill_(o.fill)
    assert bool((o.wide == o.fill).all()), f"{what}: written outside the output"
    ops = (2 * (steps + 8) + 1) * F32 * size
    near = (got - want).abs() <= ops + HALF_ULP[out] * (want.abs() + ops) + TINY[out]
    if not bool(near.all()):
        i = tuple((~near).nonzero()[0].tolist())
        raise AssertionError(f"{what}: {int((~near).sum())} of {near.numel()} differ, first at {i}: "
                             f"{float(got[i])!r} against {float(want[i])!r}")


@pytest.mark.parametrize("m,n,k,kernel", PRODUCTS)
def test_product(m, n, k, kernel):
    note(f"mxfp4 product {m}x{n}x{k}")
    g = gen(m + n + k)
    qa, sa, a = four_bits(g, m, k, 16 * (m % 2))
    qb, sb, b = four_bits(g, n, k, 16 * (n % 2))
    bias = torch.randn(n, generator=g, device=DEV) * 10
    y, size = a @ b.t(), a.abs() @ b.abs().t() + bias.abs().double()
    for out, with_bias, relu, pad, shift in (("bf16", True, True, 0, 0), ("bf16", False, False, 3, 1),
                                             ("f32", False, True, 3, 1), ("f32", True, False, 0, 0)):
        want = y + bias.double() if with_bias else y
        want = want.clamp(min=0) if relu else want
        o = Output(m, n, TYPES[out], pad, shift)
        P.cc_matmul_mxfp4(qa, sa, qb, sb, o.t, bias=bias if with_bias else None, relu=relu)
        check(o, want, size, -(-k // 64), out, f"{m}x{n}x{k} {out}")


@pytest.mark.parametrize("m,n", [(3, 5), (300, 300), (2_100, 1_281), (3_000, 3_001)])
def test_products_of_no_columns(m, n):
    """k = 0: the bias, by every kernel."""
    note(f"mxfp4 product {m}x{n}x0")
    none = [torch.empty(rows, 0, dtype=torch.uint8, device=DEV) for rows in (m, n)]
    bias = torch.randn(n, device=DEV)
    out = torch.full((m, n), 7.0, device=DEV)
    P.cc_matmul_mxfp4(none[0], none[0], none[1], none[1], out, bias=bias)
    assert torch.equal(out, bias.expand(m, n))


@pytest.mark.parametrize("m,n,k,kernel", [p for p in PRODUCTS if p[0] * p[1] < 12_000_000])
def test_equal_calls_give_equal_bits(m, n, k, kernel):
    note(f"mxfp4 product again {m}x{n}x{k}")
    g = gen(m)
    qa, sa, _ = four_bits(g, m, k)
    qb, sb, _ = four_bits(g, n, k)
    first, again = torch.empty(m, n, device=DEV), torch.empty(m, n, device=DEV)
    P.cc_matmul_mxfp4(qa, sa, qb, sb, first)
    for _ in range(3):
        P.cc_matmul_mxfp4(qa, sa, qb, sb, again)
        assert torch.equal(first, again)


@pytest.mark.parametrize("m,n,k", INSIDE + OUTSIDE)
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_linear(m, n, k, dtype):
    """Rows put in 4 bits by the product's kernel, or by a launch before it: the product of the rows that
    cc_quantize_mxfp4 gives, in 64 bits."""
    note(f"mxfp4 linear {m}x{n}x{k} {dtype}")
    g = gen(m + n + k)
    x = torch.randn(m, k + 3, generator=g, device=DEV).to(TYPES[dtype])[:, :k]
    w = torch.randn(n, k, generator=g, device=DEV)
    room = [torch.empty(rows, -(-k // 128) * 64, dtype=torch.uint8, device=DEV) for rows in (m, n)]
    scales = [torch.empty(rows, -(-k // 512) * 16, dtype=torch.uint8, device=DEV) for rows in (m, n)]
    P.cc_quantize_mxfp4(x, room[0], scales[0])
    P.cc_quantize_mxfp4(w, room[1], scales[1])
    a, b = values(room[0], scales[0]), values(room[1], scales[1])
    bias = torch.randn(n, generator=g, device=DEV)
    o = Output(m, n, TYPES[dtype])
    ws = torch.empty(P.cc_linear_mxfp4_workspace_bytes(m, n, k), dtype=torch.uint8, device=DEV)
    P.cc_linear_mxfp4(x, room[1], scales[1], o.t, bias=bias, workspace=ws)
    check(o, a @ b.t() + bias.double(), a.abs() @ b.abs().t() + bias.abs().double(), -(-k // 64), dtype,
          f"{m}x{n}x{k} {dtype}")


def test_rows_that_lie_far_apart():
    """Row strides of more than 2^24 bytes take the kernel with 64-bit offsets, whatever the size; offsets
    past 32 bits in rows, values, scales and output."""
    note("mxfp4 far rows")
    m, n, k = 270, 600, 640
    g = gen(5)
    qa, sa, a = four_bits(g, m, k)
    qb, sb, b = four_bits(g, n, k)
    wide = torch.empty((m - 1) * ((1 << 24) + 16) + 1024, dtype=torch.uint8, device=DEV)
    far = wide.as_strided((m, k // 2), ((1 << 24) + 16, 1))
    far.copy_(qa)
    far_scales = wide[512:].as_strided((m, 32), ((1 << 24) + 16, 1))
    far_scales.copy_(sa)
    o = Output(m, n, torch.float32)
    P.cc_matmul_mxfp4(far, far_scales, qb, sb, o.t)
    check(o, a @ b.t(), a.abs() @ b.abs().t(), -(-k // 64), "f32", "far rows")
    x = torch.randn(m, k, generator=g, device=DEV)
    q, s = torch.empty_like(qa), torch.empty_like(sa)
    P.cc_quantize_mxfp4(x, q, s)
    near_q, near_s = torch.empty_like(q), torch.empty_like(s)
    P.cc_quantize_mxfp4(x, far, near_s)
    P.cc_quantize_mxfp4(x, near_q, far_scales)
    assert torch.equal(far, q) and torch.equal(far_scales, s)
    assert torch.equal(near_q, q) and torch.equal(near_s, s)
    out, far_out = torch.empty_like(x), wide[1024 - 4 * 64:].view(torch.float32)
    P.cc_dequantize_mxfp4(q, s, out)
    far_out = far_out.as_strided((m, 64), ((1 << 22) + 4, 1))
    P.cc_dequantize_mxfp4(q[:, :64], s[:, :16], far_out)
    assert torch.equal(far_out, out[:, :64])


@pytest.mark.parametrize("m,n,k", [s for s in INSIDE if -(-s[0] // 16) * -(-s[1] // 16) <= 512] + OUTSIDE)
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_a_linear_layer_is_its_two_calls(m, n, k, dtype):
    """Bit by bit where both take the same kernel: everywhere but at rows put in 4 bits within the product and
    more than 512 tiles of 16 x 16, of which the product alone takes 64 x 64."""
    note(f"mxfp4 linear as two calls {m}x{n}x{k} {dtype}")
    g = gen(m + n + k)
    x = torch.randn(m, k + 3, generator=g, device=DEV).to(TYPES[dtype])[:, :k]
    w = torch.randn(n, k, generator=g, device=DEV)
    room = [torch.empty(rows, -(-k // 128) * 64, dtype=torch.uint8, device=DEV) for rows in (m, n)]
    scales = [torch.empty(rows, -(-k // 512) * 16, dtype=torch.uint8, device=DEV) for rows in (m, n)]
    P.cc_quantize_mxfp4(x, room[0], scales[0])
    P.cc_quantize_mxfp4(w, room[1], scales[1])
    bias = torch.randn(n, generator=g, device=DEV)
    one, two = (torch.empty(m, n, dtype=TYPES[dtype], device=DEV) for _ in range(2))
    ws = torch.empty(P.cc_linear_mxfp4_workspace_bytes(m, n, k), dtype=torch.uint8, device=DEV)
    P.cc_linear_mxfp4(x, room[1], scales[1], one, bias=bias, relu=True, workspace=ws)
    P.cc_matmul_mxfp4(room[0], scales[0], room[1], scales[1], two, bias=bias, relu=True)
    assert torch.equal(one, two)


@pytest.mark.parametrize("m,n,k", [(16, 300, 640), (333, 1_030, 384), (300, 9_001, 256), (512, 32_768, 256)])
def test_scales_at_both_ends(m, n, k):
    """Rows with scales of 2^-127 to 2^127, of which products reach every size of 32 bits: scales of both are
    taken together before anything is rounded, subnormal sums are kept. Each of the additions that `check`
    counts is off by a unit of 2^-149 at least; sums beyond 2^126 may pass the type's end on their way."""
    note(f"mxfp4 ends of scales {m}x{n}x{k}")
    g = gen(m + n + k)
    q, s, _ = zip(*(four_bits(g, rows, k) for rows in (m, n)))
    for i, rows in enumerate((m, n)):
        s[i].copy_(torch.randint(0, 255, (rows, 1), generator=g, device=DEV).to(torch.uint8).expand_as(s[i]))
    a, b = (values(q[i], s[i]) for i in range(2))
    want, size = a @ b.t(), a.abs() @ b.abs().t()
    out = torch.empty(m, n, device=DEV)
    P.cc_matmul_mxfp4(q[0], s[0], q[1], s[1], out)
    steps = -(-k // 64) + 8
    bound = (2 * steps + 1) * F32 * size + steps * TINY["f32"]
    inside = size < 2.0 ** 126
    assert bool(((out.double() - want).abs() <= bound)[inside].all())
    small, middle = (size < 2.0 ** -126) & (want != 0), (size > 2.0 ** -20) & (size < 2.0 ** 20)
    assert bool(small.any()) and bool(middle.any())
