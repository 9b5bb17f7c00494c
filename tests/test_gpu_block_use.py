"""The block calls in use: the example's gradients, its serving path, HIP graphs that share workspaces, two
streams at a time, and the native marshalling against the Python checks."""
from __future__ import annotations

import importlib.util
from pathlib import Path

import pytest
import torch

import paper_2609_22441_amd as P
from gpu_common import note
from layers_common import DEV
from paper_2609_22441_amd import binding as B
from paper_2609_22441_amd import layers as Y

pytestmark = pytest.mark.gpu
BF16, F16, F32, U8 = torch.bfloat16, torch.float16, torch.float32, torch.uint8


def example():
    path = Path(__file__).resolve().parents[1] / "examples" / "block.py"
    spec = importlib.util.spec_from_file_location("block_example", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_the_example_runs(capsys):
    note("block example")
    example().main()
    out = capsys.readouterr().out
    assert "step 7" in out and "serving: (4000, 512)" in out


def test_the_examples_gradients():
    """Against torch's automatic gradient of the block in 64 bits with f and the gate as the block rounded
    them: the operator's own error is a few roundings of bf16 (2^-8 relative to the largest of a row);
    products in 32 bits after it add less."""
    note("block example gradients")
    E = example()
    block = E.Block(96, DEV)
    x, h = E.hidden(50, 96, DEV)
    f, gate, _, _ = block.forward(x, h)
    g = torch.Generator(device=DEV).manual_seed(4)
    dh, dy = torch.randn(50, 96, generator=g, device=DEV).bfloat16(), torch.randn(50, 96, generator=g,
                                                                                  device=DEV)
    dx, d_h, grads = block.backward(x, h, f, gate, dh, dy)
    leaves = {n: t.double().cpu().requires_grad_() for n, t in (
        ("x", x), ("f", f), ("gate", gate), ("post", block.post), ("pre", block.pre))}
    n = torch.nn.functional.layer_norm(leaves["f"], (96,), eps=1e-5) * leaves["post"]
    y = leaves["x"] + E.SCALE * torch.sigmoid(leaves["gate"]) * n
    out = torch.nn.functional.rms_norm(y, (96,), eps=1e-6) * leaves["pre"]
    ((out * dh.double().cpu()).sum() + (y * dy.double().cpu()).sum()).backward()

    def near(got, want):
        got = got.double().cpu()
        assert bool(((got - want).abs() <= 2.0 ** -8 * want.abs().max()).all())

    near(dx, leaves["x"].grad)
    near(grads["post"], leaves["post"].grad)
    near(grads["pre"], leaves["pre"].grad)
    hd, df = h.double().cpu(), leaves["f"].grad * (f > 0).double().cpu()
    near(grads["w"], df.t() @ hd)
    near(grads["b"], df.sum(0))
    near(grads["u"], leaves["gate"].grad.t() @ hd)
    near(d_h, df @ block.w.double().cpu() + leaves["gate"].grad @ block.u.double().cpu())


def test_serving_is_its_calls_one_by_one():
    """In place and in one go against separate outputs, the values of the 4-bit weights in 64 bits."""
    note("block serving")
    E = example()
    block = E.Block(160, DEV)
    for rows in (1, 3, 70, 700):
        x, h = E.hidden(rows, 160, DEV, seed=rows)
        s = E.Serving(block)
        y, out = s(x.clone(), h)
        values = {}
        for name in ("w", "u"):
            values[name] = torch.empty(160, 160, device=DEV)
            P.cc_dequantize_mxfp4(*getattr(s, name), values[name])
        hq, hs = E.Serving.four_bits(h.float())
        hv = torch.empty(rows, 160, device=DEV)
        P.cc_dequantize_mxfp4(hq, hs, hv)
        f = torch.relu(hv.double() @ values["w"].double().t())
        u = hv.double() @ values["u"].double().t()
        # Sums in 32 bits differ from 64 by far less than half a unit of bf16, which rounds them.
        f, u = f.float().bfloat16(), u.float().bfloat16()
        want_y, want_h = torch.empty_like(x), torch.empty_like(h)
        P.cc_block_norm(f, want_y, x=x, gate=u, h=want_h, **block.norms())
        assert bool(((y - want_y).abs() <= 2.0 ** -6 * want_y.abs().max()).all())
        assert bool(((out.float() - want_h.float()).abs() <= 2.0 ** -6 * want_h.float().abs().max()).all())


class Step:
    """A training step and a serving layer on fixed buffers."""

    def __init__(self, n, cols, ws=None, lw=None):
        def e(*shape, dtype=BF16):
            return torch.zeros(*shape, dtype=dtype, device=DEV)
        self.x, self.y, self.dy, self.dx = (e(n, cols, dtype=F32) for _ in range(4))
        self.f, self.gate, self.h, self.dh, self.df, self.dgate, self.out = (e(n, cols) for _ in range(7))
        self.weights = [torch.ones(cols, device=DEV) for _ in range(2)]
        self.sums = [e(cols, dtype=F32) for _ in range(2)]
        self.q, self.s = e(cols, -(-cols // 128) * 64, dtype=U8), e(cols, -(-cols // 512) * 16, dtype=U8)
        size = P.cc_block_norm_grad_workspace_bytes(n, cols)
        self.ws = torch.empty(size, dtype=U8, device=DEV) if ws is None else ws[:size]
        size = P.cc_linear_mxfp4_workspace_bytes(n, cols, cols)
        self.lw = torch.empty(size, dtype=U8, device=DEV) if lw is None else lw[:size]

    def inputs(self, seed):
        g = torch.Generator(device=DEV).manual_seed(seed)
        for t in (self.x, self.dy, self.f, self.gate, self.dh):
            t.copy_(torch.randn(t.shape, generator=g, device=DEV))
        P.cc_quantize_mxfp4(torch.randn(self.q.shape[0], self.x.shape[1], generator=g, device=DEV),
                            self.q, self.s)

    def run(self):
        P.cc_block_norm(self.f, self.y, x=self.x, gate=self.gate, h=self.h, scale=0.5,
                        post_weight=self.weights[0], pre_weight=self.weights[1])
        P.cc_linear_mxfp4(self.h, self.q, self.s, self.out, relu=True, workspace=self.lw)
        P.cc_block_norm_grad(self.f, self.df, self.ws, x=self.x, gate=self.gate, scale=0.5,
                             post_weight=self.weights[0], pre_weight=self.weights[1], dy=self.dy,
                             dh=self.dh, dx=self.dx, dgate=self.dgate, d_post_weight=self.sums[0],
                             d_pre_weight=self.sums[1])

    def results(self):
        return [t.clone() for t in (self.y, self.h, self.out, self.df, self.dx, self.dgate, *self.sums)]

    def clear(self):
        for t in (self.y, self.h, self.out, self.df, self.dx, self.dgate, *self.sums):
            t.fill_(7)


def captured(step):
    step.inputs(0)
    step.run()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(s):
        graph.capture_begin()
        step.run()
        graph.capture_end()
    torch.cuda.current_stream().wait_stream(s)
    return graph


@pytest.mark.parametrize("n,cols", [(700, 256), (9, 1_000), (40, 17_000), (600, 4_096)])
def test_graphs_that_share_workspaces(n, cols):
    """Two captured steps on one workspace, replayed in turn with new inputs and eager work between; every
    replay against the eager call, bit by bit."""
    note(f"block graphs {n}x{cols}")
    first = Step(n, cols)
    second = Step(max(1, n // 2), cols, first.ws, first.lw)
    graphs = [captured(first), captured(second)]
    for seed in range(1, 4):
        for step, graph in zip((first, second), graphs):
            step.inputs(seed)
            step.run()
            want = step.results()
            step.clear()
            graph.replay()
            torch.cuda.synchronize()
            for a, b in zip(step.results(), want):
                assert torch.equal(a, b)


def test_two_streams_at_a_time():
    note("block streams")
    steps = [Step(3_000, 512), Step(2_500, 512)]
    want = []
    for i, step in enumerate(steps):
        step.inputs(i)
        step.run()
        want.append(step.results())
        step.clear()
    streams = [torch.cuda.Stream() for _ in steps]
    torch.cuda.synchronize()
    for _ in range(5):
        for step, s in zip(steps, streams):
            with torch.cuda.stream(s):
                step.run()
    torch.cuda.synchronize()
    for step, w in zip(steps, want):
        for a, b in zip(step.results(), w):
            assert torch.equal(a, b)


# ---- native marshalling ----

def r(*shape, dtype=F32):
    g = torch.Generator().manual_seed(sum(shape))
    if dtype == U8:
        return torch.randint(110, 130, shape, generator=g).to(U8).to(DEV)
    return torch.randn(*shape, generator=g).to(dtype).to(DEV)


def z(*shape, dtype=F32):
    return torch.zeros(*shape, dtype=dtype, device=DEV)


def calls():
    """name, positional arguments, keyword arguments, the output (an argument's number or a keyword)."""
    wide = r(40, 80, dtype=BF16)
    ws = z(P.cc_block_norm_grad_workspace_bytes(40, 24), dtype=U8)
    lw = z(P.cc_linear_mxfp4_workspace_bytes(40, 20, 600), dtype=U8)
    return [
        ("cc_block_norm", (wide[:, :24], z(40, 24)),
         dict(x=r(40, 24), gate=r(40, 24, dtype=BF16), h=z(40, 24, dtype=BF16), post_weight=r(24),
              post_bias=r(24), pre_weight=r(24), pre_bias=r(24), scale=2, post_norm=P.CC_NORM_LAYER), 1),
        ("cc_block_norm", (wide[:, :24], z(40, 30, dtype=BF16)[:, :24]), {}, 1),
        ("cc_block_norm_grad", (wide[:, :24], z(40, 24, dtype=BF16), ws),
         dict(x=r(40, 24), gate=wide[:, 30:54], dy=r(40, 24), dh=r(40, 24, dtype=BF16), dx=z(40, 24),
              dgate=z(40, 24, dtype=BF16), post_weight=r(24), post_bias=r(24), pre_weight=r(24),
              pre_bias=r(24), d_post_weight=z(24), d_post_bias=z(24), d_pre_weight=z(24),
              d_pre_bias=z(24), gate_kind=P.CC_GATE_LINEAR, accumulate=True), 1),
        ("cc_block_norm_grad", (r(40, 24, dtype=F16), z(40, 24, dtype=F16), ws),
         dict(dy=r(40, 24, dtype=F16), d_post_weight=z(24)), 1),
        ("cc_quantize_mxfp4", (r(40, 200, dtype=F16), z(40, 128, dtype=U8), z(40, 16, dtype=U8)), {}, 1),
        ("cc_dequantize_mxfp4", (r(40, 128, dtype=U8), r(40, 16, dtype=U8), z(40, 200)), {}, 2),
        ("cc_matmul_mxfp4", (r(40, 320, dtype=U8), r(40, 32, dtype=U8), r(20, 320, dtype=U8),
                             r(20, 32, dtype=U8), z(40, 20)), dict(bias=r(20), relu=True), 4),
        ("cc_linear_mxfp4", (r(40, 600, dtype=F16), r(20, 320, dtype=U8), r(20, 32, dtype=U8),
                             z(40, 20, dtype=F16)), dict(workspace=lw), 3),
    ]


@pytest.mark.parametrize("case", range(8))
def test_the_native_path_makes_the_checks_call(case, monkeypatch):
    name, args, kw, at = calls()[case]
    note(f"marshal: {name} {case}")
    checked = []
    L = Y._load()
    real = getattr(L, name)
    monkeypatch.setattr(L, name, lambda *a: checked.append(a) or real(*a))
    getattr(P, name)(*args, **kw)
    native = [args[at]] + [v for v in kw.values() if isinstance(v, torch.Tensor)]
    assert checked == []                                # the checks made no call
    _, args, kw, _ = calls()[case]
    monkeypatch.setattr(L, "marshal", B._ChecksOnly())
    getattr(P, name)(*args, **kw)
    assert len(checked) == 1
    torch.cuda.synchronize()
    for a, b in zip(native, [args[at]] + [v for v in kw.values() if isinstance(v, torch.Tensor)]):
        assert torch.equal(a, b) or a.dtype == U8


@pytest.mark.parametrize("case", range(8))
def test_every_output_is_the_checks(case, monkeypatch):
    """All tensors of a call but its workspace, those of 8 bits too."""
    name = calls()[case][0]
    note(f"marshal outputs: {name} {case}")
    got = []
    for path in (Y._load().marshal, B._ChecksOnly()):
        name, args, kw, _ = calls()[case]
        monkeypatch.setattr(Y._load(), "marshal", path)
        getattr(P, name)(*args, **kw)
        tensors = [t for i, t in enumerate(args) if not (name == "cc_block_norm_grad" and i == 2)]
        got.append(tensors + [t for key, t in kw.items()
                              if key != "workspace" and isinstance(t, torch.Tensor)])
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(*got))


@pytest.mark.parametrize("case", range(8))
def test_streams(case):
    """Work goes to the current stream, or to the one named by object or handle."""
    name, args, kw, at = calls()[case]
    note(f"marshal streams: {name} {case}")
    getattr(P, name)(*args, **kw)
    torch.cuda.synchronize()
    want = args[at].clone()
    s = torch.cuda.Stream()
    for how in ("current", "object", "handle"):
        _, args, kw, _ = calls()[case]
        s.wait_stream(torch.cuda.current_stream())
        if how == "current":
            with torch.cuda.stream(s):
                getattr(P, name)(*args, **kw)
        else:
            getattr(P, name)(*args, stream=s if how == "object" else s.cuda_stream, **kw)
        s.synchronize()
        assert torch.equal(args[at], want), how


def bad_values(a):
    yield a.cpu()                                       # host memory
    yield a[:-1]                                        # too short
    yield a.double() if a.dtype == F32 else a.float()
    if a.dim() == 2:
        yield a.repeat(2, 2)[::2, ::2]                  # strided


def bad_calls():
    for name, args, kw, _ in calls():
        for i, a in enumerate(args):
            for bad in bad_values(a):
                yield name, tuple(bad if j == i else x for j, x in enumerate(args)), kw
        for key, a in kw.items():
            if isinstance(a, torch.Tensor):
                for bad in bad_values(a):
                    yield name, args, dict(kw, **{key: bad})
        yield name, args, dict(kw, stream="x")
    norm = calls()[0]
    for key, bad in (("post_norm", 7), ("gate_kind", -1), ("post_eps", 0.0), ("scale", float("nan")),
                     ("gate_kind", 1 << 40), ("pre_norm", "rms")):
        yield norm[0], norm[1], dict(norm[2], **{key: bad})
    name, args, kw, _ = calls()[2]
    yield name, args, dict(kw, dh=None)
    yield name, args, dict(kw, gate=None)
    yield name, args, dict(kw, dy=None, dh=None, d_pre_weight=None, d_pre_bias=None)


def test_refusals_are_the_checks():
    note("marshal: refusals")
    L = Y._load()
    fast = L.marshal
    for name, args, kw in bad_calls():
        got = []
        for path in (fast, B._ChecksOnly()):
            L.marshal = path
            try:
                getattr(P, name)(*args, **kw)
                got.append(None)
            except (ValueError, TypeError, AttributeError, OverflowError, P.CCError) as e:
                got.append((type(e), str(e)))
            except Exception as e:                      # ctypes.ArgumentError
                got.append((type(e), str(e)))
            finally:
                L.marshal = fast
        assert got[0] == got[1], (name, got)
    torch.cuda.synchronize()
