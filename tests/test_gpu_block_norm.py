"""The norms around a block with its gate and residual sum, and their gradient, against the formulas in 64
bits with bounds on what 32 bits may differ by; types, kinds, sizes, strides, in-place use."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import block_oracle as O
from block_sizes import MANY_ROWS, NORMS
import paper_2609_22441_amd as P
from gpu_common import note
from layers_common import DEV, HALF_ULP, TINY, TYPES, Output, assert_close, on_gpu, rng, values

pytestmark = pytest.mark.gpu

VECTORS = ("post_weight", "post_bias", "pre_weight", "pre_bias")


def make(r, rows, cols, dtype="bf16", stream=None, post=O.RMS, pre=O.RMS, gate=O.SIGMOID,
         residual=True, weights=VECTORS, scale=0.5, offset=0.0, eps=1e-5):
    """(the call in 64 bits, its tensors)."""
    stream = stream or dtype
    c = dict(post_norm=post, pre_norm=O.NONE if pre is None else pre, gate_kind=gate or 0,
             scale=scale, post_eps=eps, pre_eps=2 * eps)
    t = {}
    f = torch.from_numpy(r.standard_normal((rows, cols)) + offset).to(TYPES[dtype])
    c["f"], t["f"] = f.double().numpy(), f
    if residual:
        c["x"], t["x"] = values(r, rows, cols, stream)
    if gate is not None:
        c["gate"], t["gate"] = values(r, rows, cols, dtype)
    for name in weights:
        w = torch.from_numpy((0.0 if "bias" in name else 1.0) + 0.3 * r.standard_normal(cols)).float()
        c[name], t[name] = w.double().numpy(), w
    return c, t


def options(c):
    return {k: c[k] for k in ("post_norm", "pre_norm", "gate_kind", "scale", "post_eps", "pre_eps")}


def close(got, bound, dtype, what):
    v, e = bound.v.reshape(got.shape), bound.e.reshape(got.shape)
    assert_close(got, v, e + HALF_ULP[dtype] * (np.abs(v) + e) + TINY[dtype], what)


def check_forward(c, t, dtype, stream, pre, pad=0, shift=0):
    rows, cols = c["f"].shape
    y = Output(rows, cols, TYPES[stream], pad, shift)
    h = Output(rows, cols, TYPES[dtype], pad, shift)
    moved = {k: on_gpu(v, pad, shift) if v.dim() == 2 else v.to(DEV) for k, v in t.items()}
    f = moved.pop("f")
    if not pre:
        moved = {k: v for k, v in moved.items() if not k.startswith("pre_")}
    P.cc_block_norm(f, y.t, h=h.t if pre else None, **moved, **options(c))
    want_y, want_h = O.norm(c)
    close(y.get(), want_y, stream, "y")
    if pre:
        close(h.get(), want_h, dtype, "h")


def check_grad(c, t, dtype, stream, r, pre=True, with_dy=True, pad=0, shift=0, sums=VECTORS):
    rows, cols = c["f"].shape
    dy = dh = None
    more = {}
    if with_dy:
        dy, dyt = values(r, rows, cols, stream)
        more["dy"] = on_gpu(dyt, pad, shift)
    if pre:
        dh, dht = values(r, rows, cols, dtype)
        more["dh"] = on_gpu(dht, pad, shift)
    out = dict(dx=Output(rows, cols, TYPES[stream], pad, shift),
               df=Output(rows, cols, TYPES[dtype], pad, shift))
    if "gate" in c:
        out["dgate"] = Output(rows, cols, TYPES[dtype], pad, shift)
    vectors = {"d_" + v: torch.full((cols,), -77.0, device=DEV) for v in sums
               if pre or not v.startswith("pre_")}
    moved = {k: on_gpu(v, pad, shift) if v.dim() == 2 else v.to(DEV) for k, v in t.items()}
    f = moved.pop("f")
    size = P.cc_block_norm_grad_workspace_bytes(rows, cols)
    ws = torch.full((size + 64,), 77, dtype=torch.uint8, device=DEV)
    P.cc_block_norm_grad(f, out["df"].t, ws[:size], **moved, **more, **options(c), **vectors,
                         **{k: v.t for k, v in out.items() if k != "df"})
    want = O.norm_grad(c, dy, dh)
    for k, o in out.items():
        close(o.get(), want[k], stream if k == "dx" else dtype, k)
    for k, v in vectors.items():
        close(v.double().cpu().numpy(), want[k], "f32", k)
    assert bool((ws[size:] == 77).all())


TYPE_PAIRS = [("bf16", "bf16"), ("bf16", "f32"), ("f16", "f16"), ("f16", "f32"), ("f32", "f32")]

@pytest.mark.parametrize("rows,cols", NORMS)
def test_sizes(rows, cols):
    note(f"block norm {rows}x{cols}")
    for i, (dtype, stream) in enumerate(TYPE_PAIRS):
        r = rng(cols * 10 + i)
        c, t = make(r, rows, cols, dtype, stream, post=O.LAYER if i % 2 else O.RMS,
                    pre=O.RMS if i % 2 else O.LAYER, gate=O.LINEAR if i == 2 else O.SIGMOID)
        check_forward(c, t, dtype, stream, True)
        check_grad(c, t, dtype, stream, r)


@pytest.mark.parametrize("post", [O.NONE, O.RMS, O.LAYER])
@pytest.mark.parametrize("pre", [None, O.NONE, O.RMS, O.LAYER])
@pytest.mark.parametrize("gate", [None, O.LINEAR, O.SIGMOID])
@pytest.mark.parametrize("residual", [False, True])
def test_kinds(post, pre, gate, residual):
    note(f"block norm kinds {post} {pre} {gate} {residual}")
    for rows, cols, dtype, stream in ((23, 104, "bf16", "f32"), (5, 1_500, "f32", "f32"),
                                      (3, 17_000, "f16", "f16")):
        r = rng(cols)
        c, t = make(r, rows, cols, dtype, stream, post, pre, gate, residual)
        check_forward(c, t, dtype, stream, pre is not None)
        check_grad(c, t, dtype, stream, r, pre is not None)


@pytest.mark.parametrize("weights", [(), ("post_weight",), ("post_bias", "pre_weight"), ("pre_bias",)])
def test_absent_vectors(weights):
    note(f"block norm weights {weights}")
    for cols in (61, 640, 18_000):
        r = rng(cols)
        c, t = make(r, 9, cols, weights=weights, post=O.LAYER)
        check_forward(c, t, "bf16", "bf16", True)
        check_grad(c, t, "bf16", "bf16", r, with_dy=False, sums=("post_bias", "pre_weight"))
        check_grad(c, t, "bf16", "bf16", r, sums=())


@pytest.mark.parametrize("dtype,stream", TYPE_PAIRS)
@pytest.mark.parametrize("pad,shift", [(0, 1), (8, 0), (3, 2), (8, 8)])
def test_strides_and_alignment(dtype, stream, pad, shift):
    note(f"block norm {dtype} {stream} pad={pad} shift={shift}")
    for rows, cols in ((11, 96), (6, 640), (3, 2_048), (2, 16_400)):
        r = rng(cols + pad)
        c, t = make(r, rows, cols, dtype, stream)
        check_forward(c, t, dtype, stream, True, pad, shift)
        check_grad(c, t, dtype, stream, r, pad=pad, shift=shift)


@pytest.mark.parametrize("rows,cols", NORMS)
def test_without_biases(rows, cols):
    """Instantiations of their own."""
    note(f"block norm without biases {rows}x{cols}")
    for i, (dtype, stream) in enumerate(TYPE_PAIRS):
        r = rng(cols * 10 + 5 + i)
        c, t = make(r, rows, cols, dtype, stream, post=O.RMS if i % 2 else O.LAYER,
                    weights=("post_weight", "pre_weight"))
        check_forward(c, t, dtype, stream, True)
        check_grad(c, t, dtype, stream, r, sums=("post_weight", "pre_weight"))


@pytest.mark.parametrize("rows,cols", MANY_ROWS)
@pytest.mark.parametrize("weights", [VECTORS, ("post_weight", "pre_weight")])
def test_many_rows(rows, cols, weights):
    """More rows than a launch has groups of lanes."""
    note(f"block norm many rows {rows}x{cols}")
    for stream in ("bf16", "f32"):
        r = rng(rows)
        c, t = make(r, rows, cols, "bf16", stream, post=O.LAYER, weights=weights)
        check_forward(c, t, "bf16", stream, True)
        check_grad(c, t, "bf16", stream, r, sums=weights)


def test_offsets_past_32_bits():
    """Rows 2^23 bytes apart, the last ones beyond 4 GiB: the same bits as of dense rows."""
    note("block norm far rows")
    rows, step = 520, (1 << 22) + 8
    for cols in (104, 2_048, 17_000):
        r = rng(cols)
        c, t = make(r, rows, cols, "bf16", "bf16", post=O.LAYER)
        moved = {k: v.to(DEV) for k, v in t.items()}
        f = moved.pop("f")
        wide = torch.empty((rows - 1) * step + cols, dtype=torch.bfloat16, device=DEV)
        far = wide.as_strided((rows, cols), (step, 1))
        y, h, far_h = torch.empty_like(f), torch.empty_like(f), torch.empty_like(f)
        P.cc_block_norm(f, y, h=h, **moved, **options(c))
        far.copy_(f)
        P.cc_block_norm(far, y, h=far_h, **moved, **options(c))
        assert torch.equal(h, far_h)
        P.cc_block_norm(f, far, h=far_h, **moved, **options(c))
        assert torch.equal(far, y)
        ws = torch.empty(P.cc_block_norm_grad_workspace_bytes(rows, cols), dtype=torch.uint8, device=DEV)
        dh, df, far_df = torch.randn_like(f), torch.empty_like(f), torch.empty_like(f)
        P.cc_block_norm_grad(f, df, ws, dh=dh, **moved, **options(c))
        far.copy_(f)
        P.cc_block_norm_grad(far, far_df, ws, dh=dh, **moved, **options(c))
        assert torch.equal(df, far_df)
        P.cc_block_norm_grad(f, far, ws, dh=dh, **moved, **options(c))
        assert torch.equal(df, far)


def test_rows_far_from_zero():
    """A mean of 300 standard deviations: squares of differences, not a difference of squares."""
    note("block norm offset")
    for cols in (100, 2_000, 17_000):
        r = rng(cols)
        c, t = make(r, 6, cols, "f32", post=O.LAYER, pre=O.LAYER, offset=300.0, gate=None)
        check_forward(c, t, "f32", "f32", True)
        check_grad(c, t, "f32", "f32", r)


def test_a_gate_far_from_zero():
    """Sigmoids at both ends: neither exp nor 1 - g loses what is left."""
    note("block norm gate ends")
    for cols in (96, 17_000):
        r = rng(cols)
        c, t = make(r, 8, cols, "f32")
        u = torch.from_numpy(np.repeat([[-200.0], [-88.0], [-30.0], [-5.0], [5.0], [30.0], [88.0], [200.0]],
                                       cols, axis=1) + r.random((8, cols))).float()
        c["gate"], t["gate"] = u.double().numpy(), u
        check_forward(c, t, "f32", "f32", True)
        check_grad(c, t, "f32", "f32", r)


def test_zero_rows_and_constant_rows():
    note("block norm zero rows")
    for cols in (40, 3_000, 17_000):
        r = rng(cols)
        for post in (O.RMS, O.LAYER):
            c, t = make(r, 4, cols, "bf16", post=post, pre=O.LAYER, residual=False, eps=1e-3)
            for row, v in ((1, 0.0), (2, 3.0)):
                t["f"][row] = v
            c["f"] = t["f"].double().numpy()
            check_forward(c, t, "bf16", "bf16", True)
            check_grad(c, t, "bf16", "bf16", r)


def test_a_nan_stays_in_its_row():
    note("block norm nan")
    for cols in (96, 1_000, 17_000):
        r = rng(cols)
        c, t = make(r, 5, cols, "f32")
        y, h = torch.empty(5, cols, device=DEV), torch.empty(5, cols, device=DEV)
        t["f"][1, 3], t["f"][3, 5] = float("nan"), float("inf")
        moved = {k: v.to(DEV) for k, v in t.items()}
        f = moved.pop("f")
        P.cc_block_norm(f, y, h=h, **moved, **options(c))
        df = torch.empty_like(f)
        ws = torch.empty(P.cc_block_norm_grad_workspace_bytes(5, cols), dtype=torch.uint8, device=DEV)
        P.cc_block_norm_grad(f, df, ws, dy=y, dh=torch.ones_like(f), **moved, **options(c))
        for out in (y, h, df):
            bad = torch.isnan(out).any(1).cpu().tolist()
            assert bad == [False, True, False, True, False]
            assert bool(torch.isfinite(out[::2]).all())


def test_infinite_elements_where_no_norm_meets_them():
    """Without norms elements are on their own: an infinity stays where it is."""
    note("block norm infinity without norms")
    for cols in (96, 17_000):
        r = rng(cols)
        c, t = make(r, 3, cols, "f32", post=O.NONE, pre=O.NONE, gate=None, weights=())
        t["f"][1, 3] = float("inf")
        moved = {k: v.to(DEV) for k, v in t.items()}
        f = moved.pop("f")
        d = torch.ones_like(f)
        df, dx = torch.empty_like(f), torch.empty_like(f)
        ws = torch.empty(P.cc_block_norm_grad_workspace_bytes(3, cols), dtype=torch.uint8, device=DEV)
        P.cc_block_norm_grad(f, df, ws, dy=d, dh=d, dx=dx, **moved, **options(c))
        assert bool((dx == 2.0).all()) and bool((df == 1.0).all())


@pytest.mark.parametrize("cols", [96, 1_000, 4_096, 17_000])
def test_in_place(cols):
    note(f"block norm in place {cols}")
    r = rng(cols)
    c, t = make(r, 13, cols, "bf16", "f32", post=O.LAYER)
    moved = {k: v.to(DEV) for k, v in t.items()}
    f = moved.pop("f")
    y, h = torch.empty_like(moved["x"]), torch.empty_like(f)
    P.cc_block_norm(f, y, h=h, **moved, **options(c))
    here = dict(moved, x=moved["x"].clone())
    g = f.clone()
    P.cc_block_norm(g, here["x"], h=g, **here, **options(c))
    assert torch.equal(here["x"], y) and torch.equal(g, h)
    size = P.cc_block_norm_grad_workspace_bytes(13, cols)
    ws = torch.empty(size, dtype=torch.uint8, device=DEV)
    dy, dh = torch.randn_like(y), torch.randn_like(f)
    dx, df = torch.empty_like(dy), torch.empty_like(dh)
    P.cc_block_norm_grad(f, df, ws, dy=dy, dh=dh, dx=dx, **moved, **options(c))
    P.cc_block_norm_grad(f, dh, ws, dy=dy, dh=dh, dx=dy, **moved, **options(c))
    assert torch.equal(dy, dx) and torch.equal(dh, df)


def test_accumulate_no_rows_and_equal_bits():
    note("block norm accumulate")
    for rows, cols in ((700, 96), (300, 1_000), (20, 17_000)):
        r = rng(rows)
        c, t = make(r, rows, cols, post=O.LAYER)
        moved = {k: v.to(DEV) for k, v in t.items()}
        f = moved.pop("f")
        d = torch.randn_like(f)
        ws = torch.empty(P.cc_block_norm_grad_workspace_bytes(rows, cols), dtype=torch.uint8, device=DEV)

        def run(sums, **kw):
            P.cc_block_norm_grad(f, torch.empty_like(f), ws, dy=d, dh=d, **moved, **options(c), **kw,
                                 **{"d_" + n: s for n, s in zip(VECTORS, sums)})

        first = [torch.empty(cols, device=DEV) for _ in VECTORS]
        again = [torch.empty(cols, device=DEV) for _ in VECTORS]
        run(first)
        ws.random_()
        run(again)
        assert all(torch.equal(a, b) for a, b in zip(first, again))
        base = [torch.randn(cols, device=DEV) for _ in VECTORS]
        added = [b.clone() for b in base]
        run(added, accumulate=True)
        for a, b, s in zip(added, base, first):
            # Up to 17 more additions of the workgroup's sums to what was there.
            size = b.abs() + s.abs() + 4 * rows ** 0.5
            assert bool(((a - b - s).abs() <= 20 * 2.0 ** -24 * size).all())
    nothing = torch.empty(0, 64, device=DEV)
    sums = [torch.full((64,), 5.0, device=DEV) for _ in VECTORS]
    kw = dict(dy=nothing, dh=nothing, **{"d_" + n: s for n, s in zip(VECTORS, sums)})
    P.cc_block_norm_grad(nothing, nothing, None, accumulate=True, **kw)
    assert all(bool((s == 5.0).all()) for s in sums)
    P.cc_block_norm_grad(nothing, nothing, None, **kw)
    assert all(bool((s == 0.0).all()) for s in sums)
    P.cc_block_norm(nothing, nothing, h=nothing)


def test_gradient_against_differences():
    """df, dx, dgate and the vectors' gradients against central differences of the call itself."""
    note("block norm differences")
    r = rng(5)
    c, t = make(r, 4, 24, "f32", post=O.LAYER, pre=O.RMS)
    moved = {k: v.to(DEV) for k, v in t.items()}
    gy, gh = (torch.from_numpy(r.standard_normal((4, 24))).float().to(DEV) for _ in range(2))
    names = ("f", "x", "gate") + VECTORS

    def loss(tensors):
        y, h = torch.empty(4, 24, device=DEV), torch.empty(4, 24, device=DEV)
        rest = {k: v for k, v in tensors.items() if k != "f"}
        P.cc_block_norm(tensors["f"], y, h=h, **rest, **options(c))
        return float((y.double() * gy).sum() + (h.double() * gh).sum())

    grads = {k: torch.empty_like(moved[k]) for k in names}
    ws = torch.empty(P.cc_block_norm_grad_workspace_bytes(4, 24), dtype=torch.uint8, device=DEV)
    rest = {k: v for k, v in moved.items() if k != "f"}
    P.cc_block_norm_grad(moved["f"], grads["f"], ws, dy=gy, dh=gh, dx=grads["x"], dgate=grads["gate"],
                         **{"d_" + v: grads[v] for v in VECTORS}, **rest, **options(c))
    # A step of 2^-6 leaves a third derivative's part, about 2^-12 of terms of size 1 to 10, and the
    # outputs' rounding, 96 elements of 2^-24 * 4 over a step of 2^-5: 2^-11.
    step = 2.0 ** -6
    for name in names:
        flat = moved[name].reshape(-1)
        for at in r.choice(flat.numel(), 6, replace=False):
            old = float(flat[at])
            flat[at] = old + step
            up = loss(moved)
            flat[at] = old - step
            down = loss(moved)
            flat[at] = old
            got = float(grads[name].reshape(-1)[at])
            assert abs((up - down) / (2 * step) - got) <= 2.0 ** -7, (name, at)
