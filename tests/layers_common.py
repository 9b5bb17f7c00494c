"""Helpers of the GPU tests of the scoring model's input layer."""
from __future__ import annotations

import numpy as np
import torch

DEV = torch.device("cuda:0")
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
F32 = 2.0 ** -24                       # half a unit in the last place, relative
HALF_ULP = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
TINY = {"f32": 2.0 ** -149, "f16": 2.0 ** -25, "bf16": 2.0 ** -133}   # subnormal results


def rng(seed):
    return np.random.default_rng(seed)


def values(r, rows, cols, dtype):
    """Random values that the type holds exactly, as float64, and their tensor."""
    t = torch.from_numpy(r.standard_normal((rows, cols))).to(TYPES[dtype])
    return t.double().numpy(), t


def on_gpu(t, pad=0, shift=0, fill=float("nan")):
    """t in GPU memory as a view into rows of `pad` more elements, `shift` elements in; what lies
    around it is `fill`."""
    rows, cols = t.shape
    wide = torch.full((rows * (cols + pad) + shift + pad,), fill, dtype=t.dtype, device=DEV) \
        if t.dtype.is_floating_point else \
        torch.full((rows * (cols + pad) + shift + pad,), 77, dtype=t.dtype, device=DEV)
    view = wide[shift:shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    view.copy_(t)
    return view


class Output:
    """An output view inside a buffer whose other elements must stay as they are."""

    def __init__(self, rows, cols, dtype, pad=0, shift=0, fill=-77.0):
        self.fill = fill
        self.wide = torch.full((rows * (cols + pad) + shift + pad + 8,), fill, dtype=dtype,
                               device=DEV)
        self.t = self.wide[shift:shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]

    def get(self):
        torch.cuda.synchronize()
        got = self.t.double().cpu().numpy()
        self.t.fill_(self.fill)
        assert bool((self.wide == self.fill).all()), "written outside the output"
        return got


def assert_close(got, want, tolerance, what=""):
    bad = ~(np.abs(got - want) <= tolerance) & ~((got == want) | (np.isnan(got) & np.isnan(want)))
    if bad.any():
        i = tuple(np.argwhere(bad)[0])
        raise AssertionError(f"{what}: {bad.sum()} of {bad.size} differ, first at {i}: "
                             f"{got[i]!r} against {want[i]!r}")
