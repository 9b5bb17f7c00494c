"""The layer calls in use: wide rows of every type, a HIP graph, offsets past 32 bits, and the example
that runs them together on joined rows."""
from __future__ import annotations

import importlib.util
from pathlib import Path

import numpy as np
import pytest
import torch

import layers_oracle as O
import paper_2609_22441_amd as P
from gpu_common import note
from layers_common import DEV, F32, HALF_ULP, TINY, TYPES, Output, assert_close, on_gpu, rng, values

pytestmark = pytest.mark.gpu

DROP = dict(p=0.25, seed=99, site=1, first_row=(1 << 32) - 1_000)


def tolerance(want, terms, out):
    return 3 * F32 * terms + HALF_ULP[out] * (np.abs(want) + 3 * F32 * terms) + TINY[out]


# Rows of 64 column blocks and more are shared out by wavefront once a call is large enough; of 8
# segments of 64 blocks, differently again.
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("rows,cols", [(5_300, 800), (4_200, 1_003), (1_100, 4_096), (1_030, 4_090)])
@pytest.mark.parametrize("pad", [0, 8, 3])
def test_wide_rows(dtype, rows, cols, pad):
    note(f"wide rows {rows}x{cols} {dtype} pad={pad}")
    r = rng(cols)
    x, t = values(r, rows, cols, dtype)
    res, rt = values(r, rows, cols, dtype)
    want = O.dropout(x, DROP, res)
    o = Output(rows, cols, TYPES[dtype], pad)
    P.cc_dropout(on_gpu(t, pad), o.t, residual=on_gpu(rt, pad), **DROP)
    terms = np.abs(O.dropout(x, DROP)) + np.abs(res)
    assert_close(o.get(), want, tolerance(want, terms, dtype), "dropout")
    ids = r.integers(-1, 40, rows)
    want = O.lookup(x[:40], ids, 0.7, DROP)
    o = Output(rows, cols, TYPES[dtype], pad)
    P.cc_embedding_lookup(on_gpu(t[:40], pad), torch.from_numpy(ids).to(DEV), o.t, scale=0.7, **DROP)
    assert_close(o.get(), want, tolerance(want, np.abs(want), dtype), "lookup")


def test_a_graph_replays_the_calls():
    """A step's calls captured once and replayed with new inputs, each replay against the same calls
    made eagerly, with eager work in between."""
    note("layers in a graph")
    n, rows, cols, out_cols = 6_000, 300, 96, 256
    ids = torch.empty(n, dtype=torch.int64, device=DEV)
    table = torch.empty(rows, cols, device=DEV)
    looked, hidden = (torch.empty(n, cols, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    grad, out = torch.empty_like(table), torch.empty(n, out_cols, dtype=torch.bfloat16, device=DEV)
    w = torch.randint(-127, 128, (out_cols, cols), device=DEV).to(torch.int8)
    sw = torch.rand(out_cols, device=DEV) / 127
    ws = torch.empty(P.cc_embedding_grad_workspace_bytes(n, rows, cols), dtype=torch.uint8, device=DEV)
    lw = torch.empty(P.cc_linear_i8_workspace_bytes(n, out_cols, cols), dtype=torch.uint8, device=DEV)
    drop = dict(p=0.1, seed=5, site=2)

    def step():
        P.cc_embedding_lookup(table, ids, looked, **drop)
        P.cc_dropout(looked, hidden, 0.2, 6)
        P.cc_linear_i8(hidden, w, sw, out, relu=True, workspace=lw)
        P.cc_embedding_grad(ids, hidden, grad, ws, **drop)

    def inputs(seed):
        g = torch.Generator(device=DEV).manual_seed(seed)
        ids.copy_(torch.randint(-1, rows, (n,), generator=g, device=DEV))
        table.copy_(torch.randn(rows, cols, generator=g, device=DEV))

    inputs(0)
    step()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(s):
        with torch.cuda.graph(graph, stream=s):
            step()
    torch.cuda.synchronize()
    for rep in range(4):
        inputs(10 + rep)
        ws.fill_(rep)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (looked, hidden, out, grad)]
        for t in (looked, hidden, out, grad):
            t.fill_(7)
        step()
        torch.cuda.synchronize()
        for a, b in zip(got, (looked, hidden, out, grad)):
            assert torch.equal(a, b), f"replay {rep}"


def test_rows_past_32_bits():
    """Byte offsets past 2^32 and element counts past 2^31, by the rows at the far end."""
    note("layers past 32 bits")
    rows, cols = 70_000, 32_768                        # 4.6 GB
    table = torch.zeros(rows, cols, dtype=torch.bfloat16, device=DEV)
    last = torch.arange(cols, device=DEV, dtype=torch.float32) % 251
    table[-1], table[-2] = last.bfloat16(), 3
    ids = torch.tensor([rows - 1, 0, rows - 2, rows], device=DEV)
    out = torch.full((4, cols), 9, dtype=torch.bfloat16, device=DEV)
    P.cc_embedding_lookup(table, ids, out)
    torch.cuda.synchronize()
    assert torch.equal(out[0], last.bfloat16()) and (out[2] == 3).all()
    assert (out[1] == 0).all() and (out[3] == 0).all()
    P.cc_dropout(table, table, 0.5, 3)                 # in place
    keep = torch.from_numpy(O.kept(2, cols, 0.5, 3, first_row=rows - 2)).to(DEV)
    torch.cuda.synchronize()
    assert torch.equal(table[-1], torch.where(keep[1], 2 * last, 0.0).bfloat16())
    assert torch.equal(table[-2], torch.where(keep[0], 6.0, 0.0).bfloat16())
    grad = torch.ones(5, cols, dtype=torch.bfloat16, device=DEV)
    ws = torch.empty(P.cc_embedding_grad_workspace_bytes(5, rows, cols), dtype=torch.uint8, device=DEV)
    P.cc_embedding_grad(torch.tensor([rows - 1, 1, rows - 1, -1, rows - 2], device=DEV), grad, table,
                        ws)
    torch.cuda.synchronize()
    assert (table[-1] == 2).all() and (table[-2] == 1).all() and (table[1] == 1).all()
    assert (table[0] == 0).all() and (table[rows // 2] == 0).all()
    a = torch.full((rows, 16), 1, dtype=torch.int8, device=DEV)
    b = torch.full((cols, 16), 2, dtype=torch.int8, device=DEV)
    a[-1], b[-1] = 3, -5
    ones = torch.ones(rows, device=DEV)
    P.cc_matmul_i8(a, ones, b, ones[:cols], table)
    torch.cuda.synchronize()
    assert (table[0, :-1] == 32).all() and (table[-1, :-1] == 96).all()
    assert float(table[-1, -1]) == -240 and float(table[-2, -1]) == -80


def example():
    path = Path(__file__).resolve().parents[1] / "examples" / "input_layer.py"
    spec = importlib.util.spec_from_file_location("input_layer", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_the_example_learns_and_serves():
    """Training against the same steps in torch with the oracle's masks, loss falling; serving against
    the product in 32 bits."""
    note("example: input layer")
    E = example()
    rows, slots = E.joined_rows(DEV, viewers=2, candidates=500)
    n, cols = rows.shape
    t = E.Training(rows, slots)
    table = torch.zeros_like(t.table)
    losses = []
    for number in range(4):
        losses.append(float(t.step(number)))
        seed = t.seed << 32 | number
        m0, m1 = (torch.from_numpy(O.kept(n, cols, E.P_DROP, seed, site)).to(DEV) for site in (0, 1))
        f = 65536 / O.threshold(E.P_DROP)
        pos = torch.where(m0, table[slots] * f, 0.0).bfloat16()
        hidden = (torch.where(m1, rows.float() * f, 0.0) + pos.float()).bfloat16()
        error = hidden.float() @ t.head - t.target
        d = (error[:, None] * t.head).bfloat16().float()
        g = torch.zeros_like(table).index_add_(0, slots, torch.where(m0, d * f, 0.0))
        table -= 0.5 * g / torch.bincount(slots, minlength=E.S_MAX + 1)[:, None]
        assert abs(losses[-1] - float(error.square().mean())) <= 1e-3 * losses[-1]
    assert torch.allclose(t.table, table, rtol=1e-3, atol=1e-3)
    assert losses[-1] < losses[0]
    weights = torch.randn(64, cols, device=DEV) / cols ** 0.5
    bias = torch.randn(64, device=DEV)
    out = E.Serving(t.table, weights, bias)(rows, slots)
    hidden = rows + t.table[slots].bfloat16()
    plain = torch.relu(hidden.float() @ weights.t() + bias)
    # Each factor of a product is rounded by at most half a step of 1/127 of its row's largest.
    step = hidden.float().abs().amax(1)[:, None] / 254 * weights.abs().sum(1) + \
        hidden.float().abs().sum(1)[:, None] * weights.abs().amax(1) / 254
    assert ((out.float() - plain).abs() <= 1.02 * step + 2.0 ** -8 * plain + 1e-6).all()


def test_gradient_of_a_table_of_more_rows_than_a_launch_has_workgroups_of_64():
    """2^30 rows and some: the rows that no id points at are written in longer strips."""
    note("grad: 2^30 rows")
    rows = (1 << 30) + 77
    ids = torch.tensor([rows - 1, 0, 1 << 29, rows, 0], device=DEV)
    dout = torch.tensor([[1.0], [2.0], [4.0], [8.0], [16.0]], device=DEV, dtype=torch.bfloat16)
    grad = torch.ones(rows, 1, device=DEV, dtype=torch.bfloat16)
    ws = torch.empty(P.cc_embedding_grad_workspace_bytes(5, rows, 1), dtype=torch.uint8, device=DEV)
    P.cc_embedding_grad(ids, dout, grad, ws)
    assert [float(grad[i]) for i in (0, 1 << 29, rows - 1)] == [18.0, 4.0, 1.0]
    assert int(grad.view(torch.int16).count_nonzero()) == 3
