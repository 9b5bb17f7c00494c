"""CPU checks of the scoring model's input layer: the header and the binding agree, host-checkable
arguments are refused before anything touches a device, the binding's checks of tensors, and the pins
of the oracle that the GPU tests compare with."""
from __future__ import annotations

import ctypes
import re
from pathlib import Path

import numpy as np
import pytest
import torch

import layers_oracle as O
from paper_2609_22441_amd import binding as B
from paper_2609_22441_amd import layers as Y
from test_binding_checks import OnGpu

ROOT = Path(__file__).resolve().parents[1]
BAD = B.CC_ERR_INVALID_ARGUMENT


# ---- the C interface ----

def test_header_and_library_declare_the_binding_surface():
    text = (ROOT / "include" / "cc_layers.h").read_text()
    declared = set(re.findall(r"^CC_API\s+[\w\s\*]*?\b(cc_\w+)\s*\(", text, flags=re.M))
    assert declared == set(Y.EXPORTS)
    lib = ctypes.CDLL(str(B.LIB_PATH))
    for name in declared:
        assert hasattr(lib, name), name
    for name, value in (("CC_F32", Y.CC_F32), ("CC_F16", Y.CC_F16), ("CC_BF16", Y.CC_BF16)):
        assert int(re.search(rf"#define {name} (\d+)", text).group(1)) == value


def caller(name, base):
    """The entry point with `base` arguments (addresses that nothing reads), some replaced."""
    f = getattr(Y._load(), name)

    def call(**kw):
        assert set(kw) <= set(base)
        return f(*dict(base, **kw).values())
    return call


NAN = float("nan")
DROPOUT_REFUSALS = [dict(p=-0.1), dict(p=1.1), dict(p=NAN), dict(first_row=-1),
                    dict(first_row=(1 << 63) - 5)]


def test_lookup_refuses():
    call = caller("cc_embedding_lookup", dict(
        table=0x10000, rows=50, table_stride=64, table_type=2, ids=0x20000, id_bytes=8, n=10,
        cols=32, scale=1.0, p=0.5, seed=1, site=0, first_row=0, out=0x30000, out_stride=64,
        out_type=2, stream=None))
    for kw in DROPOUT_REFUSALS + [
            dict(rows=-1), dict(n=-1), dict(cols=0), dict(cols=-3), dict(cols=(1 << 24) + 1),
            dict(table_type=3), dict(table_type=-1), dict(out_type=3), dict(out_type=0),
            dict(out_type=1), dict(id_bytes=2), dict(id_bytes=0), dict(table=None), dict(ids=None),
            dict(out=None), dict(table=0x10001), dict(ids=0x20004), dict(out=0x30001),
            dict(table_stride=62), dict(table_stride=65), dict(table_stride=-64),
            dict(out_stride=0), dict(out_stride=63), dict(n=1 << 62), dict(rows=1 << 60),
            dict(out=0x10000 + 49 * 64), dict(out=0x20000 + 48), dict(table_stride=1 << 62)]:
        assert call(**kw) == BAD, kw
    nothing = dict(n=0, table=None, ids=None, out=None)
    assert call(**nothing) == 0
    assert call(**nothing, cols=0) == BAD                    # still checked


def test_grad_refuses():
    need = Y.cc_embedding_grad_workspace_bytes(5000, 500, 32)
    assert need > 0
    call = caller("cc_embedding_grad", dict(
        ids=0x200000, id_bytes=8, n=5000, grad=0x300000, grad_stride=64, grad_type=2, cols=32,
        scale=1.0, p=0.5, seed=1, site=0, first_row=0, rows=500, table=0x400000, table_stride=128,
        table_type=0, accumulate=0, workspace=0x500000, workspace_bytes=need, stream=None))
    for kw in DROPOUT_REFUSALS + [
            dict(n=-1), dict(n=1 << 31), dict(rows=-1), dict(rows=(1 << 31) - 1), dict(cols=0),
            dict(grad_type=3), dict(table_type=1), dict(grad_type=0, table_type=2),
            dict(id_bytes=1), dict(ids=None), dict(ids=0x200002), dict(grad=None),
            dict(grad=0x300001), dict(table=None), dict(table=0x400002), dict(table_stride=126),
            dict(grad_stride=60), dict(workspace=None), dict(workspace=0x500008),
            dict(workspace_bytes=need - 1), dict(table=0x300000), dict(table=0x200000),
            dict(table=0x500000), dict(workspace=0x300000), dict(workspace=0x200000)]:
        assert call(**kw) == BAD, kw
    assert call(rows=0, table=None) == 0
    assert call(n=0, ids=None, grad=None, accumulate=1) == 0
    for sizes in ((-1, 5, 8), (5, -1, 8), (5, 5, 0), (1 << 31, 5, 8), (5, (1 << 31) - 1, 8)):
        assert Y.cc_embedding_grad_workspace_bytes(*sizes) == 0, sizes
    assert Y.cc_embedding_grad_workspace_bytes(5, 0, 8) == 0


def test_grad_workspace_holds_the_pairs_and_stays_small():
    for n, rows, cols in ((1, 1, 1), (2_049, 1_000, 96), (131_072, 50_000, 2_048), (500_000, 2, 16),
                          ((1 << 31) - 1, (1 << 31) - 2, 8)):
        size = Y.cc_embedding_grad_workspace_bytes(n, rows, cols)
        assert size >= 8 * n or n <= 4096 or rows <= 128      # pairs in LDS
        assert size <= 16 * n + 2 * 4 * 8 * (n // 8 + 1) * (cols // 8 + 1) + (1 << 21), (n, rows, cols)


def test_dropout_refuses():
    call = caller("cc_dropout", dict(
        x=0x10000, x_stride=64, res=0x20000, res_stride=64, n=10, cols=32, type=2, p=0.5, seed=1,
        site=0, first_row=0, out=0x30000, out_stride=64, stream=None))
    for kw in DROPOUT_REFUSALS + [
            dict(n=-1), dict(cols=0), dict(type=3), dict(x=None), dict(out=None), dict(x=0x10001),
            dict(res=0x20001), dict(out=0x30001), dict(x_stride=62), dict(res_stride=62),
            dict(out_stride=62), dict(out_stride=65), dict(out=0x10000, out_stride=66),
            dict(out=0x10002), dict(out=0x20000 + 64), dict(n=1 << 60)]:
        assert call(**kw) == BAD, kw
    assert call(n=0, x=None, out=None) == 0


def test_quantize_refuses():
    call = caller("cc_quantize_rows", dict(
        x=0x10000, x_stride=200, type=2, n=10, cols=100, q=0x20000, q_stride=112, scales=0x30000,
        stream=None))
    for kw in [dict(n=-1), dict(n=1 << 31), dict(cols=0), dict(type=4), dict(x=None), dict(q=None),
               dict(scales=None), dict(x=0x10001), dict(q=0x20008), dict(q_stride=96),
               dict(q_stride=120), dict(scales=0x30002), dict(x_stride=198), dict(q=0x10000),
               dict(scales=0x10010), dict(scales=0x20040)]:
        assert call(**kw) == BAD, kw
    assert call(n=0, x=None, q=None, scales=None) == 0


def test_product_refuses():
    call = caller("cc_matmul_i8", dict(
        a=0x10000, a_stride=96, a_scales=0x20000, b=0x30000, b_stride=112, b_scales=0x40000,
        bias=0x50000, m=10, n=20, k=96, relu=1, out=0x60000, out_stride=40, out_type=2,
        workspace=None, workspace_bytes=0, stream=None))
    for kw in [dict(m=-1), dict(n=-1), dict(k=-16), dict(k=100), dict(k=131_072), dict(m=1 << 31),
               dict(n=1 << 31), dict(out_type=3), dict(a=None), dict(b=None), dict(out=None),
               dict(a_scales=None), dict(b_scales=None), dict(a=0x10008), dict(b=0x30004),
               dict(a_stride=80), dict(a_stride=104), dict(b_stride=88), dict(out=0x60001),
               dict(out_stride=38), dict(out_stride=41), dict(a_scales=0x20001),
               dict(b_scales=0x40002), dict(bias=0x50003), dict(out=0x10000), dict(out=0x30000),
               dict(out=0x20000), dict(out=0x40000), dict(out=0x50000)]:
        assert call(**kw) == BAD, kw
    assert call(m=0, a=None, out=None) == 0
    assert call(n=0, b=None, out=None) == 0


def test_linear_refuses():
    need = Y.cc_linear_i8_workspace_bytes(10, 20, 90)
    call = caller("cc_linear_i8", dict(
        x=0x10000, x_stride=180, type=2, w=0x30000, w_stride=96, w_scales=0x40000, bias=0x50000,
        m=10, n=20, k=90, relu=1, out=0x60000, out_stride=40, workspace=0x70000,
        workspace_bytes=need, stream=None))
    for kw in [dict(m=-1), dict(n=-1), dict(k=0), dict(k=131_057), dict(type=3), dict(x=None),
               dict(w=None), dict(w_scales=None), dict(out=None), dict(workspace=None),
               dict(workspace_bytes=need - 1), dict(workspace=0x70008), dict(x=0x10001),
               dict(x_stride=178), dict(w_stride=80), dict(w_stride=90), dict(out=0x10000),
               dict(out=0x70000), dict(workspace=0x10000), dict(workspace=0x30000),
               dict(workspace=0x40000), dict(workspace=0x50000)]:
        assert call(**kw) == BAD, kw
    assert call(m=0, x=None, out=None) == 0
    for sizes in ((0, 5, 5), (5, 0, 5), (5, 5, 0), (-1, 5, 5), (1 << 31, 5, 5), (5, 5, 131_057)):
        assert Y.cc_linear_i8_workspace_bytes(*sizes) == 0, sizes


# ---- the binding ----

class Stub:
    """The library: sizes from the real one, calls recorded."""

    def __init__(self):
        real = Y._load()
        self.calls = []
        for k in ("codes", "id_bytes", "i8", "f32"):
            setattr(self, k, getattr(real, k))
        self.marshal = B._ChecksOnly()
        self.current_device = lambda: 0
        for name in Y.EXPORTS:
            setattr(self, "at_" + name, 0)
            if name.endswith("_bytes"):
                setattr(self, name, getattr(real, name))
            else:
                setattr(self, name, lambda *a, name=name: self.calls.append((name, a)) or 0)


class At(OnGpu):
    """A host tensor that reports a place on GPU `device`."""

    def __init__(self, t, device=0):
        super().__init__(t)
        self.device_index = device

    def get_device(self):
        return self.device_index

    def view(self, *shape):
        return At(self.t.view(*shape), self.device_index)


@pytest.fixture
def stub(monkeypatch):
    s = Stub()
    monkeypatch.setattr(Y, "_layers", s)
    return s


def g(*shape, dtype=torch.float32, device=0):
    return At(torch.zeros(*shape, dtype=dtype), device)


I64, I32, I8, BF16, F16 = torch.int64, torch.int32, torch.int8, torch.bfloat16, torch.float16


def lookup_args():
    return dict(table=g(50, 24, dtype=BF16), ids=g(10, dtype=I64), out=g(10, 24, dtype=BF16))


def grad_args():
    return dict(ids=g(5000, dtype=I32), grad_out=g(5000, 24, dtype=BF16), grad_table=g(50, 24),
                workspace=g(1 << 20, dtype=torch.uint8))


def dropout_args():
    return dict(x=g(10, 24), out=g(10, 24), residual=g(10, 24), p=0.5, seed=3)


def quantize_args():
    return dict(x=g(10, 24, dtype=F16), q=g(10, 32, dtype=I8), scales=g(10))


def matmul_args():
    return dict(a=g(10, 32, dtype=I8), a_scales=g(10), b=g(20, 32, dtype=I8), b_scales=g(20),
                out=g(10, 20, dtype=BF16), bias=g(20))


def linear_args():
    return dict(x=g(10, 30), w=g(20, 32, dtype=I8), w_scales=g(20), out=g(10, 20), bias=g(20),
                workspace=g(1 << 12, dtype=torch.uint8))


CALLS = {"cc_embedding_lookup": lookup_args, "cc_embedding_grad": grad_args,
         "cc_dropout": dropout_args, "cc_quantize_rows": quantize_args,
         "cc_matmul_i8": matmul_args, "cc_linear_i8": linear_args}


@pytest.mark.parametrize("name", CALLS)
def test_valid_calls_reach_the_library(stub, name):
    getattr(Y, name)(**CALLS[name](), stream=0)
    assert [c[0] for c in stub.calls] == [name]


def test_rows_of_wider_tensors_and_of_more_dimensions(stub):
    wide = torch.zeros(10, 80)
    Y.cc_dropout(At(wide[:, :24]), At(torch.zeros(2, 5, 24)), 0.1, 1, stream=0)
    (_, a), = stub.calls
    assert a[1] == 320 and a[4] == 10 and a[5] == 24 and a[-2] == 96


STRIDED = At(torch.zeros(24, 10).t())
EXPANDED = At(torch.zeros(1, 24).expand(10, 24))
REFUSALS = [
    ("cc_embedding_lookup", "table", torch.zeros(50, 24, dtype=BF16), ValueError, "GPU memory"),
    ("cc_embedding_lookup", "table", g(50, 24, dtype=I64), TypeError, "float32"),
    ("cc_embedding_lookup", "table", g(24, 50, dtype=BF16), ValueError, "50 columns"),
    ("cc_embedding_lookup", "table", g(50, 24, dtype=BF16, device=1), ValueError, "one device"),
    ("cc_embedding_lookup", "ids", g(10, dtype=torch.int16), TypeError, "int64 or int32"),
    ("cc_embedding_lookup", "ids", g(9, dtype=I64), ValueError, "9 rows"),
    ("cc_embedding_lookup", "ids", At(torch.zeros(20, dtype=I64)[::2]), ValueError, "contiguous"),
    ("cc_embedding_lookup", "out", g(10, 24, dtype=F16), TypeError, "bfloat16"),
    ("cc_embedding_lookup", "out", At(torch.zeros(24, 10, dtype=BF16).t()), ValueError, "dense"),
    ("cc_embedding_lookup", "p", 1.5, ValueError, "p: must lie"),
    ("cc_embedding_lookup", "p", NAN, ValueError, "p: must lie"),
    ("cc_embedding_lookup", "site", 1 << 32, ValueError, "site"),
    ("cc_embedding_lookup", "first_row", -1, ValueError, "first_row"),
    ("cc_embedding_grad", "grad_out", g(11, 24, dtype=BF16), ValueError, "5000 rows"),
    ("cc_embedding_grad", "grad_table", g(50, 24, dtype=F16), TypeError, "float32 or"),
    ("cc_embedding_grad", "grad_table", g(50, 23), ValueError, "23 columns"),
    ("cc_embedding_grad", "workspace", g(16, dtype=torch.uint8), ValueError, "bytes"),
    ("cc_embedding_grad", "workspace", None, ValueError, "bytes"),
    ("cc_dropout", "out", g(10, 24, dtype=BF16), TypeError, "float32"),
    ("cc_dropout", "out", g(9, 24), ValueError, "10 rows"),
    ("cc_dropout", "residual", g(10, 24, dtype=BF16), TypeError, "float32"),
    ("cc_dropout", "residual", g(10, 25), ValueError, "24 columns"),
    ("cc_dropout", "residual", EXPANDED, ValueError, "overlap"),
    ("cc_dropout", "x", STRIDED, ValueError, "dense"),
    ("cc_quantize_rows", "q", g(10, 24, dtype=I8), ValueError, "32 columns"),
    ("cc_quantize_rows", "q", g(10, 32, dtype=torch.uint8), TypeError, "int8"),
    ("cc_quantize_rows", "scales", g(9), ValueError, "10 elements"),
    ("cc_quantize_rows", "scales", g(10, dtype=BF16), TypeError, "float32"),
    ("cc_matmul_i8", "a", g(10, 32), TypeError, "int8"),
    ("cc_matmul_i8", "b", g(20, 16, dtype=I8), ValueError, "32 columns"),
    ("cc_matmul_i8", "a_scales", g(9), ValueError, "10 elements"),
    ("cc_matmul_i8", "b_scales", g(19), ValueError, "20 elements"),
    ("cc_matmul_i8", "bias", g(19), ValueError, "20 elements"),
    ("cc_matmul_i8", "out", g(10, 21, dtype=BF16), ValueError, "20 columns"),
    ("cc_matmul_i8", "out", g(11, 20, dtype=BF16), ValueError, "10 rows"),
    ("cc_linear_i8", "x", g(10, 33), ValueError, "48 columns"),
    ("cc_linear_i8", "x", g(10, 30, dtype=I8), TypeError, "float32"),
    ("cc_linear_i8", "w", g(20, 30, dtype=I8), ValueError, "32 columns"),
    ("cc_linear_i8", "out", g(10, 20, dtype=BF16), TypeError, "float32"),
    ("cc_linear_i8", "workspace", None, ValueError, "bytes"),
]


@pytest.mark.parametrize("name,arg,bad,exc,match", REFUSALS)
def test_binding_refuses(stub, name, arg, bad, exc, match):
    a = CALLS[name]()
    a[arg] = bad
    with pytest.raises(exc, match=match):
        getattr(Y, name)(**a, stream=0)
    assert stub.calls == []


def test_binding_refuses_another_current_device(stub):
    stub.current_device = lambda: 1
    with pytest.raises(ValueError, match="current device"):
        Y.cc_dropout(g(4, 8), g(4, 8), 0.5, 1, stream=0)
    assert stub.calls == []


@pytest.mark.parametrize("name", CALLS)
def test_native_marshalling_leaves_host_tensors_to_the_checks(name):
    """Host tensors are not plain: the native function answers None, and the checks word the error."""
    a = {k: v.t if isinstance(v, OnGpu) else v for k, v in CALLS[name]().items()}
    with pytest.raises(ValueError, match="GPU memory"):
        getattr(Y, name)(**a, stream=0)


def test_status_raises(stub):
    stub.cc_dropout = lambda *a: 1
    with pytest.raises(B.CCError, match="cc_dropout: CC_ERR_INVALID_ARGUMENT"):
        Y.cc_dropout(g(4, 8), g(4, 8), 0.5, 1, stream=0)


# ---- pins of the oracle ----

def test_generator_gives_the_published_words():
    """The known answers of Philox4x32-10 that its authors publish: counter and key of zeros, of ones,
    and of digits of pi."""
    assert O.philox([0] * 4, [0] * 2) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    ones = 0xFFFFFFFF
    assert O.philox([ones] * 4, [ones] * 2) == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]
    assert O.philox([0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344], [0xA4093822, 0x299F31D0]) == \
        [0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1]


def test_mask_follows_the_counters():
    p, seed, site, first = 0.37, 0xFEDC_BA98_7654_3210, 9, (1 << 32) - 3
    got = O.kept(6, 21, p, seed, site, first)
    for r in range(6):
        for c in range(21):
            w = O.philox([(first + r) & O.M32, (first + r) >> 32, c // 8, site],
                         [seed & O.M32, seed >> 32])
            bits = (w[(c % 8) // 2] >> (16 * (c % 2))) & 0xFFFF
            assert got[r, c] == (bits < O.threshold(p))


@pytest.mark.parametrize("p", [0.0, 0.1, 0.5, 0.9, 1.0])
def test_mask_keeps_its_share(p):
    """64,000 draws: the share kept lies within five standard deviations of T / 65536; masks of other
    seeds, sites and rows agree as often as independent ones."""
    t = O.threshold(p) / 65536
    a = O.kept(1000, 64, p, 1)
    assert abs(a.mean() - t) <= 5 * np.sqrt(t * (1 - t) / a.size)
    for b in (O.kept(1000, 64, p, 2), O.kept(1000, 64, p, 1, site=1),
              O.kept(1000, 64, p, 1, first_row=1000), O.kept(1000, 64, p, 1 << 32 | 1)):
        same = t * t + (1 - t) * (1 - t)
        assert abs((a == b).mean() - same) <= 5 * np.sqrt(same * (1 - same) / a.size) + 1e-12


def test_gradient_is_the_transpose_of_the_lookup():
    r = np.random.default_rng(1)
    table, w = r.standard_normal((11, 13)), r.standard_normal((40, 13))
    ids = r.integers(-1, 12, 40)
    drop = dict(p=0.3, seed=5, site=2, first_row=70)
    g, _, _ = O.grad(ids, w, 11, 1.5, drop)
    assert np.isclose((O.lookup(table, ids, 1.5, drop) * w).sum(), (g * table).sum())


def test_quantisation_rounds_within_half_a_step():
    r = np.random.default_rng(2)
    x = r.standard_normal((20, 50)).astype(np.float32)
    q, s = O.quantize(x)
    assert q.shape == (20, 64) and (q[:, 50:] == 0).all() and np.abs(q).max() == 127
    assert (np.abs(q[:, :50] * s[:, None].astype(np.float64) - x) <= 0.5001 * s[:, None]).all()
