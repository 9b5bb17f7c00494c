"""The native marshalling (csrc/marshal.c) of the block norms and 4-bit rows on the CPU: host tensors that
report GPU residency, and C functions that record their arguments. Every call is made once with the native
path in front and once through the checks alone; both reach the same function with the same arguments,
each pointer and stride in its own place."""
import ctypes

import pytest
import torch

from paper_2609_22441_amd import binding as B
from paper_2609_22441_amd import layers as Y
from test_layers_cpu import BF16, F16, At
from test_marshal_cpu import Off

F32, U8 = torch.float32, torch.uint8
STREAM = 7


class Recorder:
    """The library's functions as ones that record (name, arguments) and return 0; sizes are the real ones."""

    def __init__(self, real, marshal):
        self.calls, self.keep, self.marshal = [], [], marshal
        for k in ("codes", "id_bytes", "i8", "u8", "f32"):
            setattr(self, k, getattr(real, k))
        self.current_device = lambda: 0
        for name in Y.EXPORTS:
            f = getattr(real, name)
            if not name.endswith("_bytes"):
                f = ctypes.CFUNCTYPE(ctypes.c_int, *f.argtypes)(self.recorder(name))
                self.keep.append(f)
            setattr(self, name, f)
            setattr(self, "at_" + name, ctypes.cast(f, ctypes.c_void_p).value)

    def recorder(self, name):
        return lambda *args: self.calls.append((name, args)) or 0


@pytest.fixture
def both(monkeypatch):
    """both(name, args) makes the call on each path and returns the arguments that reached the library; the
    native path has to have made the call itself."""
    from paper_2609_22441_amd import _marshal
    real = Y._load()
    _marshal.init(At, torch.int64, torch.int8, lambda: STREAM)
    _marshal.init_layers(F32, F16, BF16, torch.int32, lambda: 0, lambda device: STREAM)
    _marshal.init_blocks(U8)
    monkeypatch.setattr(Y, "_stream", lambda s: STREAM if s is None else s)

    def run(name, args):
        got = []
        for marshal in (_marshal, Off()):
            rec = Recorder(real, marshal)
            monkeypatch.setattr(Y, "_layers", rec)
            if marshal is _marshal:
                for checked in ("_matrix", "_one_device"):           # the checks have no part in it
                    monkeypatch.setattr(Y, checked, None)
            getattr(Y, name)(**args)
            if marshal is _marshal:
                for checked, f in real_checks.items():
                    monkeypatch.setattr(Y, checked, f)
            assert [c[0] for c in rec.calls] == [name]
            got.append(rec.calls[0][1])
        return got

    real_checks = {checked: getattr(Y, checked) for checked in ("_matrix", "_one_device")}
    yield run
    _marshal.init(torch.Tensor, torch.int64, torch.int8, B._current_stream)
    _marshal.init_layers(F32, F16, BF16, torch.int32, torch._C._cuda_getDevice,
                         torch._C._cuda_getCurrentRawStream)


def m(rows, cols, dtype=F32, pad=0):
    """A matrix with rows of `pad` more elements."""
    return At(torch.zeros(rows, cols + pad, dtype=dtype)[:, :cols])


def v(n):
    return At(torch.zeros(n))


def full_norm():
    return dict(f=m(10, 24, BF16, 1), y=m(10, 24, F32, 2), x=m(10, 24, F32, 3), gate=m(10, 24, BF16, 4),
                h=m(10, 24, BF16, 5), post_weight=v(24), post_bias=v(24), pre_weight=v(24), pre_bias=v(24),
                gate_kind=0, post_norm=2, post_eps=0.25, scale=3, pre_norm=0, pre_eps=0.5)


def full_norm_grad():
    return dict(f=m(10, 24, F16, 1), df=m(10, 24, F16, 2), workspace=At(torch.zeros(1 << 20, dtype=U8)),
                x=m(10, 24, F32, 3), gate=m(10, 24, F16, 4), dy=m(10, 24, F32, 5), dh=m(10, 24, F16, 6),
                dx=m(10, 24, F32, 7), dgate=m(10, 24, F16, 8), post_weight=v(24), post_bias=v(24),
                pre_weight=v(24), pre_bias=v(24), d_post_weight=v(24), d_post_bias=v(24), d_pre_weight=v(24),
                d_pre_bias=v(24), gate_kind=1, post_norm=1, post_eps=0.25, scale=0.75, pre_norm=2, pre_eps=0.5,
                accumulate=True)


def without(args, *names, **other):
    return dict({k: a for k, a in args.items() if k not in names}, **other)


SUMS = ("d_post_weight", "d_post_bias", "d_pre_weight", "d_pre_bias")
VECTORS = ("post_weight", "post_bias", "pre_weight", "pre_bias")

CALLS = [
    ("cc_block_norm", full_norm),
    ("cc_block_norm", lambda: without(full_norm(), "x", "gate", "h", *VECTORS)),
    ("cc_block_norm", lambda: without(full_norm(), "gate", "post_bias", "pre_weight", stream=11)),
    ("cc_block_norm", lambda: dict(f=m(1, 24, pad=9), y=m(1, 24, pad=9))),
    ("cc_block_norm_grad", full_norm_grad),
    ("cc_block_norm_grad", lambda: without(full_norm_grad(), "dh", "d_pre_weight", "d_pre_bias")),
    ("cc_block_norm_grad", lambda: without(full_norm_grad(), "dy", "gate", "dgate", *SUMS)),
    ("cc_block_norm_grad", lambda: without(full_norm_grad(), "dy", "dx", "x", *VECTORS, accumulate=False)),
    ("cc_quantize_mxfp4", lambda: dict(x=m(10, 200, BF16, 1), q=m(10, 128, U8, 16), scales=m(10, 16, U8, 32))),
    ("cc_quantize_mxfp4", lambda: dict(x=m(1, 513), q=m(1, 320, U8), scales=m(1, 32, U8, 32))),
    ("cc_dequantize_mxfp4", lambda: dict(q=m(10, 128, U8, 16), scales=m(10, 16, U8, 32), out=m(10, 200, F16, 1))),
    ("cc_matmul_mxfp4", lambda: dict(a=m(10, 320, U8, 16), a_scales=m(10, 32, U8, 32), b=m(20, 320, U8, 48),
                                     b_scales=m(20, 32, U8, 64), out=m(10, 20, BF16, 1), bias=v(20), relu=True)),
    ("cc_matmul_mxfp4", lambda: dict(a=m(10, 0, U8), a_scales=m(10, 0, U8), b=m(20, 0, U8),
                                     b_scales=m(20, 0, U8), out=m(10, 20))),
    ("cc_linear_mxfp4", lambda: dict(x=m(10, 600, F16, 1), w=m(20, 320, U8, 16), w_scales=m(20, 32, U8, 32),
                                     out=m(10, 20, F16, 2), bias=v(20), relu=True,
                                     workspace=At(torch.zeros(1 << 13, dtype=U8)))),
    ("cc_linear_mxfp4", lambda: dict(x=m(3, 64), w=m(5, 64, U8), w_scales=m(5, 16, U8), out=m(3, 5, pad=3),
                                     workspace=At(torch.zeros(1 << 12, dtype=U8)), stream=11)),
]


@pytest.mark.parametrize("case", range(len(CALLS)))
def test_native_path_and_checks_make_the_same_call(both, case):
    name, args = CALLS[case]
    native, checked = both(name, args())          # of the same tensors
    assert native == checked
    pointers = [a for a, t in zip(native, getattr(Y._load(), name).argtypes) if t is ctypes.c_void_p and a]
    assert len(set(pointers)) == len(pointers)
