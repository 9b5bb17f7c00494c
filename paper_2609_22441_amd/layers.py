"""The scoring model's layers: binding of include/cc_layers.h.

Embedding lookup and its gradient, dropout from a counter-based generator, the norms around a block
with its gate and residual sum and their gradient, row quantisation and products in 8-bit integers and
in microscaled 4-bit floating point, on torch tensors in GPU memory. Argument checks and errors are those of binding.py: a
failed check raises ValueError or TypeError, a status other than CC_OK raises CCError, and nothing is
enqueued then. Matrices are [rows, columns] with dense rows and any row stride; tensors of more
dimensions are taken as [-1, last] where that is a view. Outputs and workspaces are the caller's; a
buffer that another stream has allocated needs torch's record_stream as with any other kernel.
"""
from __future__ import annotations

import ctypes

from . import binding as _b
from .binding import _check, _fail, _stream

# Every symbol that include/cc_layers.h declares.
EXPORTS = (
    "cc_embedding_lookup", "cc_embedding_grad_workspace_bytes", "cc_embedding_grad", "cc_dropout",
    "cc_quantize_rows", "cc_matmul_i8_workspace_bytes", "cc_matmul_i8",
    "cc_linear_i8_workspace_bytes", "cc_linear_i8",
    "cc_block_norm", "cc_block_norm_grad_workspace_bytes", "cc_block_norm_grad",
    "cc_quantize_mxfp4", "cc_dequantize_mxfp4", "cc_matmul_mxfp4_workspace_bytes",
    "cc_matmul_mxfp4", "cc_linear_mxfp4_workspace_bytes", "cc_linear_mxfp4",
)

CC_F32, CC_F16, CC_BF16 = 0, 1, 2
CC_NORM_NONE, CC_NORM_RMS, CC_NORM_LAYER = 0, 1, 2
CC_GATE_LINEAR, CC_GATE_SIGMOID = 0, 1
_MASK64 = (1 << 64) - 1


class _Layers:
    """The library's functions with their argument types, and torch's types by their code."""

    def __init__(self, L):
        import torch
        i64, i32, u32, u64 = ctypes.c_int64, ctypes.c_int32, ctypes.c_uint32, ctypes.c_uint64
        f64, vp, st = ctypes.c_double, ctypes.c_void_p, ctypes.c_int
        drop = [f64, u64, u32, i64]
        sig = {
            "cc_embedding_lookup": [vp, i64, i64, i32, vp, i32, i64, i32, f64, *drop, vp, i64, i32,
                                    vp],
            "cc_embedding_grad": [vp, i32, i64, vp, i64, i32, i32, f64, *drop, i64, vp, i64, i32,
                                  i32, vp, i64, vp],
            "cc_dropout": [vp, i64, vp, i64, i64, i32, i32, *drop, vp, i64, vp],
            "cc_quantize_rows": [vp, i64, i32, i64, i32, vp, i64, vp, vp],
            "cc_matmul_i8": [vp, i64, vp, vp, i64, vp, vp, i64, i64, i64, i32, vp, i64, i32, vp,
                             i64, vp],
            "cc_linear_i8": [vp, i64, i32, vp, i64, vp, vp, i64, i64, i64, i32, vp, i64, vp, i64,
                             vp],
            "cc_block_norm": [vp, i64, i32, vp, i64, vp, i64, i32, i32, i32, vp, vp, f64, i32, vp,
                              vp, f64, f64, i64, i32, vp, i64, vp, i64, vp],
            "cc_block_norm_grad": [vp, i64, i32, vp, i64, vp, i64, i32, i32, i32, vp, vp, f64, i32,
                                   vp, f64, f64, i64, i32, vp, i64, vp, i64, vp, i64, vp, i64, vp,
                                   i64, vp, vp, vp, vp, i32, vp, i64, vp],
            "cc_quantize_mxfp4": [vp, i64, i32, i64, i32, vp, i64, vp, i64, vp],
            "cc_dequantize_mxfp4": [vp, i64, vp, i64, i64, i32, vp, i64, i32, vp],
            "cc_matmul_mxfp4": [vp, i64, vp, i64, vp, i64, vp, i64, vp, i64, i64, i64, i32, vp, i64,
                                i32, vp, i64, vp],
            "cc_linear_mxfp4": [vp, i64, i32, vp, i64, vp, i64, vp, i64, i64, i64, i32, vp, i64, vp,
                                i64, vp],
            "cc_block_norm_grad_workspace_bytes": [i64, i32],
            "cc_matmul_mxfp4_workspace_bytes": [i64, i64, i64],
            "cc_linear_mxfp4_workspace_bytes": [i64, i64, i64],
            "cc_embedding_grad_workspace_bytes": [i64, i64, i32],
            "cc_matmul_i8_workspace_bytes": [i64, i64, i64],
            "cc_linear_i8_workspace_bytes": [i64, i64, i64],
        }
        for name, args in sig.items():
            f = getattr(L, name)
            f.argtypes = args
            f.restype = i64 if name.endswith("_bytes") else st
            setattr(self, name, f)
        # Native marshalling (csrc/marshal.c) of plain calls: None from it means that the checks below
        # decide. It takes function addresses.
        try:
            raw, device = torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice
            L.marshal.init_layers(torch.float32, torch.float16, torch.bfloat16, torch.int32, device,
                                  raw)
            L.marshal.init_blocks(torch.uint8)
            self.marshal = L.marshal
        except AttributeError:
            self.marshal = _b._ChecksOnly()
        for name in sig:
            setattr(self, "at_" + name, ctypes.cast(getattr(L, name), vp).value)
        self.codes = {torch.float32: CC_F32, torch.float16: CC_F16, torch.bfloat16: CC_BF16}
        self.id_bytes = {torch.int64: 8, torch.int32: 4}
        self.i8, self.f32 = torch.int8, torch.float32
        self.u8 = torch.uint8
        self.current_device = torch.cuda.current_device


_layers = None


def _load() -> _Layers:
    global _layers
    if _layers is None:
        _layers = _Layers(_b.lib())
    return _layers


def _matrix(x, name: str, width: int = 0):
    """(pointer, row stride in bytes, rows, columns) of a matrix in GPU memory."""
    if x.dim() != 2:
        if x.dim() < 1:
            _fail(name, f"must have rows (shape {tuple(x.shape)})")
        try:
            x = x.view(-1, x.shape[-1])
        except RuntimeError:
            _fail(name, f"of shape {tuple(x.shape)} is no view of rows of {x.shape[-1]}")
    rows, cols = x.shape
    step, inner = x.stride()
    if inner != 1 and cols > 1:
        _fail(name, "rows must be dense (the last dimension contiguous)")
    if rows > 1 and step < cols:
        _fail(name, f"rows must not overlap (row stride {step}, {cols} columns)")
    if not x.is_cuda:
        _fail(name, f"must be in GPU memory (is on {x.device})")
    if width and cols != width:
        _fail(name, f"needs {width} columns (shape {tuple(x.shape)})")
    size = x.element_size()
    return x.data_ptr(), (step if rows > 1 else cols) * size, rows, cols


def _type(L, x, name: str) -> int:
    code = L.codes.get(x.dtype)
    if code is None:
        _fail(name, f"must be float32, float16 or bfloat16 (is {x.dtype})", TypeError)
    return code


def _one_device(L, first, *rest) -> None:
    """Every tensor is on the current device, where the kernels run."""
    device = first.get_device()
    for x in rest:
        if x is not None and x.get_device() != device:
            _fail("tensors", "must be on one device")
    if device != L.current_device():
        _fail("tensors", f"must be on the current device (are on cuda:{device})")


def _ids(L, ids, n=None):
    size = L.id_bytes.get(ids.dtype)
    if size is None:
        _fail("ids", f"must be int64 or int32 (is {ids.dtype})", TypeError)
    return _b._arr(ids, "ids", ids.dtype), size, ids.numel()


def _mask(p: float, seed: int, site: int, first_row: int):
    if not 0.0 <= p <= 1.0:
        _fail("p", f"must lie in [0, 1] (is {p})")
    if not 0 <= site < 1 << 32:
        _fail("site", f"must lie in [0, 2^32) (is {site})")
    if not 0 <= first_row < 1 << 63:
        _fail("first_row", f"must lie in [0, 2^63) (is {first_row})")
    return p, seed & _MASK64, site, first_row


def _work(workspace, need: int):
    """(pointer, bytes) of a workspace of at least `need` bytes."""
    if workspace is None:
        if need:
            _fail("workspace", f"needs {need} bytes")
        return None, 0
    p = _b._bytes_arr(workspace, "workspace", need)
    return p, workspace.numel() * workspace.element_size()


def cc_embedding_lookup(table, ids, out, scale: float = 1.0, p: float = 0.0, seed: int = 0,
                        site: int = 0, first_row: int = 0, stream=None) -> None:
    """out[t] = table[ids[t]] * scale with dropout of probability p; an id outside the table gives
    a zero row (see include/cc_layers.h)."""
    L = _layers or _load()
    st = L.marshal.lookup(L.at_cc_embedding_lookup, table, ids, out, scale, p, seed, site,
                          first_row, stream)
    if st is not None:
        return _check(st, "cc_embedding_lookup")
    pt, table_stride, rows, cols = _matrix(table, "table")
    pi, id_bytes, n = _ids(L, ids)
    po, out_stride, out_rows, _ = _matrix(out, "out", cols)
    if out_rows != n:
        _fail("out", f"needs {n} rows, one per id (shape {tuple(out.shape)})")
    tt, to = _type(L, table, "table"), _type(L, out, "out")
    if to != tt and tt != CC_F32:
        _fail("out", f"must be {table.dtype} as the table is (is {out.dtype})", TypeError)
    _one_device(L, out, table, ids)
    _check(L.cc_embedding_lookup(pt, rows, table_stride, tt, pi, id_bytes, n, cols, scale,
                                 *_mask(p, seed, site, first_row), po, out_stride, to,
                                 _stream(stream)), "cc_embedding_lookup")


def cc_embedding_grad_workspace_bytes(n_ids: int, n_rows: int, cols: int) -> int:
    return _load().cc_embedding_grad_workspace_bytes(n_ids, n_rows, cols)


def cc_embedding_grad(ids, grad_out, grad_table, workspace, scale: float = 1.0, p: float = 0.0,
                      seed: int = 0, site: int = 0, first_row: int = 0, accumulate: bool = False,
                      stream=None) -> None:
    """grad_table[r] = the sum of grad_out's rows whose id is r, with the scale and the dropout mask
    of the lookup; with `accumulate` added to what grad_table holds. Equal calls give equal bits."""
    L = _layers or _load()
    st = L.marshal.grad(L.at_cc_embedding_grad, L.at_cc_embedding_grad_workspace_bytes, ids, grad_out,
                        grad_table, workspace, scale, p, seed, site, first_row, accumulate, stream)
    if st is not None:
        return _check(st, "cc_embedding_grad")
    pi, id_bytes, n = _ids(L, ids)
    pt, table_stride, rows, cols = _matrix(grad_table, "grad_table")
    pg, grad_stride, grad_rows, _ = _matrix(grad_out, "grad_out", cols)
    if grad_rows != n:
        _fail("grad_out", f"needs {n} rows, one per id (shape {tuple(grad_out.shape)})")
    tg, tt = _type(L, grad_out, "grad_out"), _type(L, grad_table, "grad_table")
    if tt != tg and tt != CC_F32:
        _fail("grad_table", f"must be float32 or {grad_out.dtype} (is {grad_table.dtype})",
              TypeError)
    pw, size = _work(workspace, L.cc_embedding_grad_workspace_bytes(n, rows, cols))
    _one_device(L, grad_table, grad_out, ids, workspace)
    _check(L.cc_embedding_grad(pi, id_bytes, n, pg, grad_stride, tg, cols, scale,
                               *_mask(p, seed, site, first_row), rows, pt, table_stride, tt,
                               1 if accumulate else 0, pw, size, _stream(stream)),
           "cc_embedding_grad")


def cc_dropout(x, out, p: float, seed: int, site: int = 0, first_row: int = 0, residual=None,
               stream=None) -> None:
    """out = dropout(x) (+ residual): the mask is drawn from (seed, site, first_row + row, column),
    so the same call on a gradient is the backward pass. out may be x or residual."""
    L = _layers or _load()
    st = L.marshal.dropout(L.at_cc_dropout, x, out, p, seed, site, first_row, residual, stream)
    if st is not None:
        return _check(st, "cc_dropout")
    px, x_stride, n, cols = _matrix(x, "x")
    po, out_stride, out_rows, _ = _matrix(out, "out", cols)
    if out_rows != n:
        _fail("out", f"needs {n} rows (shape {tuple(out.shape)})")
    t = _type(L, x, "x")
    if out.dtype != x.dtype:
        _fail("out", f"must be {x.dtype} as x is (is {out.dtype})", TypeError)
    pr, res_stride = None, 0
    if residual is not None:
        pr, res_stride, res_rows, _ = _matrix(residual, "residual", cols)
        if res_rows != n:
            _fail("residual", f"needs {n} rows (shape {tuple(residual.shape)})")
        if residual.dtype != x.dtype:
            _fail("residual", f"must be {x.dtype} as x is (is {residual.dtype})", TypeError)
    _one_device(L, out, x, residual)
    _check(L.cc_dropout(px, x_stride, pr, res_stride, n, cols, t,
                        *_mask(p, seed, site, first_row), po, out_stride, _stream(stream)),
           "cc_dropout")


def _padded(k: int) -> int:
    return (k + 15) // 16 * 16


def cc_quantize_rows(x, q, scales, stream=None) -> None:
    """q, scales: the rows of x in 8-bit integers and one factor per row. q has x's columns rounded
    up to a multiple of 16, the added ones zero."""
    L = _layers or _load()
    st = L.marshal.quantize(L.at_cc_quantize_rows, x, q, scales, stream)
    if st is not None:
        return _check(st, "cc_quantize_rows")
    px, x_stride, n, cols = _matrix(x, "x")
    if q.dtype != L.i8:
        _fail("q", f"must be int8 (is {q.dtype})", TypeError)
    pq, q_stride, q_rows, _ = _matrix(q, "q", _padded(cols))
    if q_rows != n:
        _fail("q", f"needs {n} rows (shape {tuple(q.shape)})")
    ps = _b._arr(scales, "scales", L.f32, n)
    t = _type(L, x, "x")
    _one_device(L, q, x, scales)
    _check(L.cc_quantize_rows(px, x_stride, t, n, cols, pq, q_stride, ps, _stream(stream)),
           "cc_quantize_rows")


def _weights(L, b, b_scales, bias, name: str, width: int):
    """(pointer, row stride, rows, scales, bias) of weights in 8 bits, one row per output."""
    if b.dtype != L.i8:
        _fail(name, f"must be int8 (is {b.dtype})", TypeError)
    pb, stride, n, _ = _matrix(b, name, width)
    ps = _b._arr(b_scales, name + "_scales", L.f32, n)
    return pb, stride, n, ps, _b._arr(bias, "bias", L.f32, n, optional=True)


def cc_matmul_i8_workspace_bytes(m: int, n: int, k: int) -> int:
    return _load().cc_matmul_i8_workspace_bytes(m, n, k)


def cc_matmul_i8(a, a_scales, b, b_scales, out, bias=None, relu: bool = False, workspace=None,
                 stream=None) -> None:
    """out = act(a b' * a_scales * b_scales + bias) for int8 a [m, k] and b [n, k], k a multiple of
    16; the integer sums are exact."""
    L = _layers or _load()
    st = L.marshal.matmul(L.at_cc_matmul_i8, L.at_cc_matmul_i8_workspace_bytes, a, a_scales, b,
                          b_scales, out, bias, relu, workspace, stream)
    if st is not None:
        return _check(st, "cc_matmul_i8")
    if a.dtype != L.i8:
        _fail("a", f"must be int8 (is {a.dtype})", TypeError)
    pa, a_stride, m, k = _matrix(a, "a")
    pas = _b._arr(a_scales, "a_scales", L.f32, m)
    pb, b_stride, n, pbs, pbias = _weights(L, b, b_scales, bias, "b", k)
    po, out_stride, out_rows, _ = _matrix(out, "out", n)
    if out_rows != m:
        _fail("out", f"needs {m} rows (shape {tuple(out.shape)})")
    t = _type(L, out, "out")
    pw, size = _work(workspace, L.cc_matmul_i8_workspace_bytes(m, n, k))
    _one_device(L, out, a, a_scales, b, b_scales, bias, workspace)
    _check(L.cc_matmul_i8(pa, a_stride, pas, pb, b_stride, pbs, pbias, m, n, k, 1 if relu else 0,
                          po, out_stride, t, pw, size, _stream(stream)), "cc_matmul_i8")


def cc_linear_i8_workspace_bytes(m: int, n: int, k: int) -> int:
    return _load().cc_linear_i8_workspace_bytes(m, n, k)


def cc_linear_i8(x, w, w_scales, out, bias=None, relu: bool = False, workspace=None,
                 stream=None) -> None:
    """out = act(x W' + bias) with x quantised row by row in the call and weights that
    cc_quantize_rows has put in 8 bits: w [n, columns of x rounded up to a multiple of 16]."""
    L = _layers or _load()
    st = L.marshal.linear(L.at_cc_linear_i8, L.at_cc_linear_i8_workspace_bytes, x, w, w_scales, out,
                          bias, relu, workspace, stream)
    if st is not None:
        return _check(st, "cc_linear_i8")
    px, x_stride, m, k = _matrix(x, "x")
    t = _type(L, x, "x")
    pw, w_stride, n, pws, pbias = _weights(L, w, w_scales, bias, "w", _padded(k))
    po, out_stride, out_rows, _ = _matrix(out, "out", n)
    if out_rows != m:
        _fail("out", f"needs {m} rows (shape {tuple(out.shape)})")
    if out.dtype != x.dtype:
        _fail("out", f"must be {x.dtype} as x is (is {out.dtype})", TypeError)
    pws_, size = _work(workspace, L.cc_linear_i8_workspace_bytes(m, n, k))
    _one_device(L, out, x, w, w_scales, bias, workspace)
    _check(L.cc_linear_i8(px, x_stride, t, pw, w_stride, pws, pbias, m, n, k, 1 if relu else 0, po,
                          out_stride, pws_, size, _stream(stream)), "cc_linear_i8")


def _like(L, x, name: str, dtype, rows: int, cols: int, of: str):
    """(pointer, row stride) of a matrix [rows, cols] of the type that `of` has, or nothing."""
    if x is None:
        return None, 0
    p, stride, n, _ = _matrix(x, name, cols)
    if n != rows:
        _fail(name, f"needs {rows} rows (shape {tuple(x.shape)})")
    if x.dtype != dtype:
        _fail(name, f"must be {dtype} as {of} is (is {x.dtype})", TypeError)
    return p, stride


def _vector(L, x, name: str, cols: int):
    """Pointer of a float vector of one element per column, or nothing."""
    return _b._arr(x, name, L.f32, cols, optional=True)


def _stream_type(L, x, f, name: str) -> int:
    """The residual stream's type: f's or float32."""
    code = _type(L, x, name)
    if x.dtype != f.dtype and code != CC_F32:
        _fail(name, f"must be {f.dtype} as f is, or float32 (is {x.dtype})", TypeError)
    return code


def cc_block_norm(f, y, x=None, gate=None, gate_kind: int = CC_GATE_SIGMOID,
                  post_norm: int = CC_NORM_RMS, post_weight=None, post_bias=None,
                  post_eps: float = 1e-6, scale: float = 1.0, h=None, pre_norm: int = CC_NORM_RMS,
                  pre_weight=None, pre_bias=None, pre_eps: float = 1e-6, stream=None) -> None:
    """y = x + scale * gate * post(f) and, with h, h = pre(y): the norm of a block's output f, its gate,
    the residual sum, and the norm that the next block begins with. y and x are of f's type or float32,
    gate and h of f's; y may be x, h may be f (see include/cc_layers.h)."""
    L = _layers or _load()
    st = L.marshal.norm(L.at_cc_block_norm, f, y, x, gate, gate_kind, post_norm, post_weight, post_bias,
                        post_eps, scale, h, pre_norm, pre_weight, pre_bias, pre_eps, stream)
    if st is not None:
        return _check(st, "cc_block_norm")
    pf, f_stride, n, cols = _matrix(f, "f")
    t, ts = _type(L, f, "f"), _stream_type(L, y, f, "y")
    py, y_stride = _like(L, y, "y", y.dtype, n, cols, "y")
    px, x_stride = _like(L, x, "x", y.dtype, n, cols, "y")
    pg, gate_stride = _like(L, gate, "gate", f.dtype, n, cols, "f")
    ph, h_stride = _like(L, h, "h", f.dtype, n, cols, "f")
    vectors = [_vector(L, v, name, cols) for v, name in (
        (post_weight, "post_weight"), (post_bias, "post_bias"), (pre_weight, "pre_weight"),
        (pre_bias, "pre_bias"))]
    _one_device(L, y, f, x, gate, h, post_weight, post_bias, pre_weight, pre_bias)
    _check(L.cc_block_norm(px, x_stride, ts, pf, f_stride, pg, gate_stride, gate_kind, t, post_norm,
                           vectors[0], vectors[1], post_eps, pre_norm, vectors[2], vectors[3],
                           pre_eps, scale, n, cols, py, y_stride, ph, h_stride, _stream(stream)),
           "cc_block_norm")


def cc_block_norm_grad_workspace_bytes(n_rows: int, cols: int) -> int:
    return _load().cc_block_norm_grad_workspace_bytes(n_rows, cols)


def cc_block_norm_grad(f, df, workspace, x=None, gate=None, gate_kind: int = CC_GATE_SIGMOID,
                       post_norm: int = CC_NORM_RMS, post_weight=None, post_bias=None,
                       post_eps: float = 1e-6, scale: float = 1.0, pre_norm: int = CC_NORM_RMS,
                       pre_weight=None, pre_bias=None, pre_eps: float = 1e-6, dy=None, dh=None,
                       dx=None, dgate=None, d_post_weight=None, d_post_bias=None,
                       d_pre_weight=None, d_pre_bias=None, accumulate: bool = False,
                       stream=None) -> None:
    """Gradients of cc_block_norm from those of y (dy) and h (dh): df, and where a tensor is given dx,
    dgate and those of weights and biases, with `accumulate` added to what these hold. The forward
    call's arguments are given again (pre_bias has no part in a gradient); dx may be dy, df may be
    dh. Equal calls give equal bits."""
    L = _layers or _load()
    st = L.marshal.norm_grad(
        L.at_cc_block_norm_grad, L.at_cc_block_norm_grad_workspace_bytes, f, df, workspace, x, gate,
        gate_kind, post_norm, post_weight, post_bias, post_eps, scale, pre_norm, pre_weight, pre_bias,
        pre_eps, dy, dh, dx, dgate, d_post_weight, d_post_bias, d_pre_weight, d_pre_bias, accumulate,
        stream)
    if st is not None:
        return _check(st, "cc_block_norm_grad")
    pf, f_stride, n, cols = _matrix(f, "f")
    t = _type(L, f, "f")
    given = [(v, name) for v, name in ((dy, "dy"), (dx, "dx"), (x, "x")) if v is not None]
    of = given[0][0].dtype if given else f.dtype
    ts = _stream_type(L, given[0][0], f, given[0][1]) if given else t
    if dy is None and dh is None:
        _fail("dy, dh", "one of them is needed")
    if dgate is not None and gate is None:
        _fail("dgate", "needs the gate")
    if dh is None and (d_pre_weight is not None or d_pre_bias is not None):
        _fail("d_pre_weight, d_pre_bias", "need dh")
    pairs = [_like(L, v, name, dtype, n, cols, other) for v, name, dtype, other in (
        (x, "x", of, "the residual stream"), (gate, "gate", f.dtype, "f"),
        (dy, "dy", of, "the residual stream"), (dh, "dh", f.dtype, "f"),
        (dx, "dx", of, "the residual stream"), (df, "df", f.dtype, "f"),
        (dgate, "dgate", f.dtype, "f"))]
    (px, x_stride), (pg, gate_stride), *grads = pairs
    vectors = [_vector(L, v, name, cols) for v, name in (
        (post_weight, "post_weight"), (post_bias, "post_bias"), (pre_weight, "pre_weight"),
        (d_post_weight, "d_post_weight"), (d_post_bias, "d_post_bias"),
        (d_pre_weight, "d_pre_weight"), (d_pre_bias, "d_pre_bias"))]
    pw, size = _work(workspace, L.cc_block_norm_grad_workspace_bytes(n, cols))
    _one_device(L, df, f, x, gate, dy, dh, dx, dgate, post_weight, post_bias, pre_weight,
                d_post_weight, d_post_bias, d_pre_weight, d_pre_bias, workspace)
    _check(L.cc_block_norm_grad(px, x_stride, ts, pf, f_stride, pg, gate_stride, gate_kind, t,
                                post_norm, vectors[0], vectors[1], post_eps, pre_norm, vectors[2],
                                pre_eps, scale, n, cols, *[v for pair in grads for v in pair],
                                *vectors[3:], 1 if accumulate else 0, pw, size, _stream(stream)),
           "cc_block_norm_grad")


def _mx_width(k: int):
    """(bytes of values, bytes of scales) of a row of k values in 4 bits."""
    return (k + 127) // 128 * 64, (k + 511) // 512 * 16


def _of_width(x, name: str, width: int):
    """As _matrix, of `width` columns also where that is 0."""
    matrix = _matrix(x, name, width)
    if matrix[3] != width:
        _fail(name, f"needs {width} columns (shape {tuple(x.shape)})")
    return matrix


def _mx(L, q, scales, name: str, k=None, rows=None):
    """(pointer, row stride, scales' pointer and row stride, rows, k) of rows in 4 bits; of k values, or
    of as many as q has."""
    for v, what in ((q, name), (scales, name + "_scales" if name != "q" else "scales")):
        if v.dtype != L.u8:
            _fail(what, f"must be uint8 (is {v.dtype})", TypeError)
    if k is None:
        k = _matrix(q, name)[3] * 2
        if k % 128:
            _fail(name, f"needs a multiple of 64 columns (shape {tuple(q.shape)})")
    width, scale_width = _mx_width(k)
    p, stride, n, _ = _of_width(q, name, width)
    what = name + "_scales" if name != "q" else "scales"
    ps, scale_stride, scale_rows, _ = _of_width(scales, what, scale_width)
    if rows is not None and n != rows:
        _fail(name, f"needs {rows} rows (shape {tuple(q.shape)})")
    if scale_rows != n:
        _fail(what, f"needs {n} rows (shape {tuple(scales.shape)})")
    return p, stride, ps, scale_stride, n, k


def cc_quantize_mxfp4(x, q, scales, stream=None) -> None:
    """q, scales: the rows of x in microscaled 4-bit floating point. q is uint8 [rows, 64 for each 128
    columns begun], two values to a byte; scales uint8 [rows, 16 for each 512 columns begun]."""
    L = _layers or _load()
    st = L.marshal.mx_quantize(L.at_cc_quantize_mxfp4, x, q, scales, stream)
    if st is not None:
        return _check(st, "cc_quantize_mxfp4")
    px, x_stride, n, cols = _matrix(x, "x")
    t = _type(L, x, "x")
    pq, q_stride, ps, scales_stride, _, _ = _mx(L, q, scales, "q", cols, n)
    _one_device(L, q, x, scales)
    _check(L.cc_quantize_mxfp4(px, x_stride, t, n, cols, pq, q_stride, ps, scales_stride,
                               _stream(stream)), "cc_quantize_mxfp4")


def cc_dequantize_mxfp4(q, scales, out, stream=None) -> None:
    """out: the values of rows in 4 bits, as many columns as out has."""
    L = _layers or _load()
    st = L.marshal.mx_dequantize(L.at_cc_dequantize_mxfp4, q, scales, out, stream)
    if st is not None:
        return _check(st, "cc_dequantize_mxfp4")
    po, out_stride, n, cols = _matrix(out, "out")
    t = _type(L, out, "out")
    pq, q_stride, ps, scales_stride, _, _ = _mx(L, q, scales, "q", cols, n)
    _one_device(L, out, q, scales)
    _check(L.cc_dequantize_mxfp4(pq, q_stride, ps, scales_stride, n, cols, po, out_stride, t,
                                 _stream(stream)), "cc_dequantize_mxfp4")


def cc_matmul_mxfp4_workspace_bytes(m: int, n: int, k: int) -> int:
    return _load().cc_matmul_mxfp4_workspace_bytes(m, n, k)


def cc_matmul_mxfp4(a, a_scales, b, b_scales, out, bias=None, relu: bool = False, workspace=None,
                    stream=None) -> None:
    """out = act(a b' + bias) for rows in 4 bits, a of m and b of n rows, as cc_quantize_mxfp4 writes
    them; sums are in 32 bits."""
    L = _layers or _load()
    st = L.marshal.mx_matmul(L.at_cc_matmul_mxfp4, L.at_cc_matmul_mxfp4_workspace_bytes, a, a_scales, b,
                             b_scales, out, bias, relu, workspace, stream)
    if st is not None:
        return _check(st, "cc_matmul_mxfp4")
    pa, a_stride, pas, as_stride, m, k = _mx(L, a, a_scales, "a")
    pb, b_stride, pbs, bs_stride, n, _ = _mx(L, b, b_scales, "b", k)
    pbias = _b._arr(bias, "bias", L.f32, n, optional=True)
    po, out_stride, out_rows, _ = _of_width(out, "out", n)
    if out_rows != m:
        _fail("out", f"needs {m} rows (shape {tuple(out.shape)})")
    t = _type(L, out, "out")
    pw, size = _work(workspace, L.cc_matmul_mxfp4_workspace_bytes(m, n, k))
    _one_device(L, out, a, a_scales, b, b_scales, bias, workspace)
    _check(L.cc_matmul_mxfp4(pa, a_stride, pas, as_stride, pb, b_stride, pbs, bs_stride, pbias, m, n,
                             k, 1 if relu else 0, po, out_stride, t, pw, size, _stream(stream)),
           "cc_matmul_mxfp4")


def cc_linear_mxfp4_workspace_bytes(m: int, n: int, k: int) -> int:
    return _load().cc_linear_mxfp4_workspace_bytes(m, n, k)


def cc_linear_mxfp4(x, w, w_scales, out, bias=None, relu: bool = False, workspace=None,
                    stream=None) -> None:
    """out = act(x W' + bias) with x put in 4 bits in the call and weights that cc_quantize_mxfp4 has put
    in 4 bits, one row per output."""
    L = _layers or _load()
    st = L.marshal.mx_linear(L.at_cc_linear_mxfp4, L.at_cc_linear_mxfp4_workspace_bytes, x, w, w_scales,
                             out, bias, relu, workspace, stream)
    if st is not None:
        return _check(st, "cc_linear_mxfp4")
    px, x_stride, m, k = _matrix(x, "x")
    t = _type(L, x, "x")
    pw, w_stride, pws, ws_stride, n, _ = _mx(L, w, w_scales, "w", k)
    pbias = _b._arr(bias, "bias", L.f32, n, optional=True)
    po, out_stride, out_rows, _ = _of_width(out, "out", n)
    if out_rows != m:
        _fail("out", f"needs {m} rows (shape {tuple(out.shape)})")
    if out.dtype != x.dtype:
        _fail("out", f"must be {x.dtype} as x is (is {out.dtype})", TypeError)
    pws_, size = _work(workspace, L.cc_linear_mxfp4_workspace_bytes(m, n, k))
    _one_device(L, out, x, w, w_scales, bias, workspace)
    _check(L.cc_linear_mxfp4(px, x_stride, t, pw, w_stride, pws, ws_stride, pbias, m, n, k,
                             1 if relu else 0, po, out_stride, pws_, size, _stream(stream)),
           "cc_linear_mxfp4")
