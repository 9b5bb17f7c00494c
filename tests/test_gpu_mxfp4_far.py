"""4-bit products whose rows lie far apart: more 16 x 16 tiles than a launch may have, and the tile kernels'
32-bit offsets up to their limit."""
from __future__ import annotations

import pytest
import torch

import paper_2609_22441_amd as P
from gpu_common import note
from layers_common import DEV, Output
from test_gpu_mxfp4_products import check, four_bits, gen, values

pytestmark = pytest.mark.gpu

STEP = 1 << 24                       # bytes between rows up to which a tile's rows have 32-bit offsets
LAUNCH = 16 * ((1 << 23) - 1)        # rows of 16 x 16 tiles side by side that a launch has room for


def far_apart(q, s, step):
    """The same rows, `step` bytes apart, values and scales of a row next to each other."""
    rows, width, scale_width = q.shape[0], q.shape[1], s.shape[1]
    assert width <= 4096 and scale_width <= 4096
    wide = torch.empty((rows - 1) * step + 8192, dtype=torch.uint8, device=DEV)
    far = wide.as_strided((rows, width), (step, 1))
    far_scales = wide[4096:].as_strided((rows, scale_width), (step, 1))
    far.copy_(q)
    far_scales.copy_(s)
    return far, far_scales


@pytest.mark.parametrize("far", ["a", "b"])
def test_more_tiles_than_a_launch_has(far):
    """Two rows over 2^24 bytes apart take the kernel of few rows whatever the others are: at over 2^27 of
    them in several launches, each result as in a call of fewer rows."""
    note(f"mxfp4 many tiles, {far} far apart")
    many, k = LAUNCH + 16 + 40, 128
    g = gen(1)
    q = torch.empty(many, 64, dtype=torch.uint8, device=DEV).random_(generator=g)
    s = torch.randint(119, 131, (many, 16), generator=g, dtype=torch.uint8, device=DEV)
    two = four_bits(g, 2, k)
    two_q, two_s = far_apart(two[0], two[1], STEP + 16)
    bias = torch.randn(2 if far == "b" else many, generator=g, device=DEV)

    def product(q, s, bias, out):
        if far == "b":
            P.cc_matmul_mxfp4(q, s, two_q, two_s, out, bias=bias)
        else:
            P.cc_matmul_mxfp4(two_q, two_s, q, s, out, bias=bias)

    shape = (lambda n: (n, 2)) if far == "b" else (lambda n: (2, n))
    of = (lambda t, i, n: t[i:i + n]) if far == "b" else (lambda t, i, n: t[:, i:i + n])
    out = torch.full(shape(many), 7.0, dtype=torch.bfloat16, device=DEV)
    product(q, s, bias, out)
    each = 1 << 24
    for i in range(0, many, each):
        n = min(each, many - i)
        part = torch.empty(shape(n), dtype=torch.bfloat16, device=DEV)
        product(q[i:i + n], s[i:i + n], bias if far == "b" else bias[i:i + n], part)
        assert torch.equal(part, of(out, i, n)), i
    # The first, the last and those around the border of the launches, in 64 bits.
    for i in (0, LAUNCH - 32, many - 64):
        v = values(q[i:i + 64], s[i:i + 64])
        y, size = v @ two[2].t(), v.abs() @ two[2].abs().t()
        add = (bias if far == "b" else bias[i:i + 64, None]).double()
        want, size = y + add, size + add.abs()
        o = Output(*shape(64), torch.bfloat16)
        o.t.copy_(of(out, i, 64))
        check(o, *((want, size) if far == "b" else (want.t(), size.t())), 2, "bf16", f"rows from {i}")


@pytest.mark.parametrize("m,n,k", [
    (333, 1_030, 2_055),             # 64 x 64
    (300, 9_001, 640),               # 128 x 128
    (512, 32_768, 256)])             # 256 x 256
@pytest.mark.parametrize("far", ["a", "b"])
def test_offsets_of_a_tile_up_to_the_limit(m, n, k, far):
    """Rows 2^24 bytes apart, the most that the tile kernels take: those of a tile lie up to 255 * 2^24 bytes
    from its first, past 2^31. The same bits as of dense rows."""
    note(f"mxfp4 far tiles {m}x{n}x{k} {far}")
    if far == "b":
        m, n = n, m
    g = gen(m + k)
    qa, sa, a = four_bits(g, m, k)
    qb, sb, b = four_bits(g, n, k)
    dense = torch.empty(m, n, device=DEV)
    P.cc_matmul_mxfp4(qa, sa, qb, sb, dense)
    if far == "a":
        qa, sa = far_apart(qa, sa, STEP)
    else:
        qb, sb = far_apart(qb, sb, STEP)
    o = Output(m, n, torch.float32)
    P.cc_matmul_mxfp4(qa, sa, qb, sb, o.t)
    assert torch.equal(o.t, dense)
    check(o, a @ b.t(), a.abs() @ b.abs().t(), -(-k // 64), "f32", f"{m}x{n}x{k} {far}")
