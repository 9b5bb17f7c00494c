"""Timed cases of a block of the scoring model: the norms after and before a block with its gate and
residual sum, their gradient, and microscaled 4-bit floating point (rows to 4 bits and back, the
product, the linear layer).

Each case is a dict of plain values. ``listed()`` names the fixed ones, ``draw(rng)`` gives more of
the same ranges, ``prepare`` makes what a caller holds before the call, ``run`` is one pass, in
elementary torch operations or, with ``own`` set, through the package's entry points; ``exact``
gives a pass's outputs in 64 bits.

Five kinds of case:
  norm     n = N(f), y = x + scale * g * n, h = N(y): N is none, rms or layer, each with a weight and
           (layer) a bias of its own; g is 1, a gate u or sigmoid(u); without a residual x, y = n
  grad     the gradient of x, f, u and of the weights from those of y and h
  round    rows to 4 bits and back: the values that the 4-bit form stands for
  linear   a linear layer on floating-point rows, put in 4 bits within the call; weights in 4 bits
  product  4-bit rows times 4-bit weights

The 4-bit form. A block of 32 values of a row has a scale 2^(s - 127) and a value each of 0, 0.5, 1,
1.5, 2, 3, 4, 6 and a sign (OCP Microscaling Formats, E2M1 with E8M0). s is the exponent (biased) of the
largest magnitude, rounded to one bit of mantissa, less 2; values are rounded to nearest, ties to
even, and at most 6. Two values to a byte, the first in the low half; rows are padded with zeros, of
values to 128, of scales to 16.
"""
from __future__ import annotations

import math

import torch

own = False
DEV = "cuda"
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}
NORMS = ("none", "rms", "layer")
GATES = ("none", "linear", "sigmoid")
GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
EPS = 1e-5
MAX_ELEMENTS = 1 << 28          # of a drawn case's largest array
MAX_MACS = 1 << 39              # of a drawn product


def listed():
    return [
        # A decoding step of a batch, one token each: both norms, gate and residual. Latency counts.
        _norm("norm", "norm_tokens", rows=64, cols=4_096, dtype="bf16"),
        # A request's 50,000 rows after the first dense layer: the layer norm of a block, alone.
        _norm("norm", "norm_request", rows=50_000, cols=512, dtype="f16", post="layer", pre="",
              gate="none", residual=False, scale=1.0),
        # A training step's hidden rows with the residual stream in 32 bits.
        _norm("norm", "norm_train", rows=65_536, cols=4_096, dtype="bf16", stream="f32"),
        # Odd in both directions, 32 bits, the gate as it is.
        _norm("grad", "grad_ragged", rows=999, cols=97, dtype="f32", post="layer", pre="layer",
              gate="linear"),
        # The backward pass of the request's layer norm.
        _norm("grad", "grad_request", rows=50_000, cols=512, dtype="bf16", post="layer", pre="",
              gate="none", residual=False, scale=1.0),
        # The backward pass of a training step's block.
        _norm("grad", "grad_train", rows=65_536, cols=4_096, dtype="bf16"),
        # A few rows of odd length in 32 bits.
        _round("round_ragged", rows=333, cols=2_055, dtype="f32"),
        # A wide layer's weights, or a large batch's rows.
        _round("round_wide", rows=16_384, cols=8_192, dtype="bf16"),
        # One token through a square layer: the weights' bytes and the launch count.
        _product("linear", "linear_token", m=1, n=4_096, k=4_096, dtype="bf16"),
        # A long prompt or a large batch through a wide layer.
        _product("linear", "linear_large", m=16_384, n=8_192, k=8_192, dtype="bf16"),
        # A few hundred rows, nothing a multiple of a tile, 32-bit output.
        _product("product", "product_ragged", m=333, n=1_030, k=2_055, dtype="f32"),
        # A wide layer of rows that are in 4 bits already.
        _product("product", "product_wide", m=8_192, n=16_384, k=4_096, dtype="bf16"),
    ]


def _norm(kind, name, rows, cols, dtype, stream=None, post="rms", pre="rms", gate="sigmoid",
          residual=True, scale=0.5, pad=0):
    return dict(name=name, kind=kind, rows=rows, cols=cols, dtype=dtype, stream=stream or dtype,
                post=post, pre=pre, gate=gate, residual=residual, scale=scale, pad=pad)


def _round(name, rows, cols, dtype, pad=0):
    return dict(name=name, kind="round", rows=rows, cols=cols, dtype=dtype, pad=pad)


def _product(kind, name, m, n, k, dtype, bias=True, relu=True, pad=0):
    return dict(name=name, kind=kind, m=m, n=n, k=k, dtype=dtype, bias=bias, relu=relu, pad=pad)


def draw(rng):
    kind = rng.choice(["norm", "grad", "round", "linear", "product"])
    while True:
        c = _DRAW[kind](rng)
        c.pop("name")
        if kind in ("linear", "product"):
            fits = c["m"] * c["n"] * c["k"] <= MAX_MACS and \
                max(c["m"] * c["n"], c["m"] * c["k"], c["n"] * c["k"]) <= MAX_ELEMENTS
        else:
            fits = c["rows"] * c["cols"] <= MAX_ELEMENTS // (2 if c["dtype"] == "f32" else 1)
        if fits:
            return c


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _cols(rng, lo=16, hi=16_384):
    """Columns: mostly multiples of 8, as models have them, some odd."""
    c = _log(rng, lo, hi)
    return c if rng.random() < 0.25 else max(8, c // 8 * 8)


def _dtype(rng):
    return rng.choice(["bf16", "bf16", "f16", "f32"])


def _draw_norm(kind):
    def make(rng):
        dtype = _dtype(rng)
        post = rng.choice(["rms", "layer", "rms", "none"])
        pre = rng.choice(["rms", "layer", "rms", ""] if post != "none" else ["rms", "layer"])
        return _norm(kind, "", rows=_log(rng, 1, 131_072), cols=_cols(rng), dtype=dtype,
                     stream=rng.choice([dtype, "f32"]), post=post, pre=pre,
                     gate=rng.choice(["sigmoid", "linear", "none"]),
                     residual=post == "none" or rng.random() < 0.8,
                     scale=rng.choice([1.0, 0.5, 0.22]), pad=rng.choice([0, 0, 8, 3]))
    return make


def _draw_round(rng):
    return _round("", rows=_log(rng, 1, 131_072), cols=_cols(rng), dtype=_dtype(rng),
                  pad=rng.choice([0, 0, 8, 3]))


def _draw_product(kind):
    def make(rng):
        return _product(kind, "", m=_log(rng, 1, 50_000), n=_cols(rng, 64), k=_cols(rng, 64),
                        dtype=_dtype(rng), bias=rng.random() < 0.7, relu=rng.random() < 0.5,
                        pad=rng.choice([0, 0, 8, 3]) if kind == "linear" else 0)
    return make


_DRAW = {"norm": _draw_norm("norm"), "grad": _draw_norm("grad"), "round": _draw_round,
         "linear": _draw_product("linear"), "product": _draw_product("product")}


# ---- inputs ----

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 1_000_003 + 29)
    return g


def _empty(rows, cols, dtype, pad=0):
    return torch.empty(rows, cols + pad, device=DEV, dtype=TYPES[dtype])[:, :cols]


def _hidden(rows, cols, dtype, g, pad=0, unit=1.0):
    """Hidden rows: normal, columns of different size, as a view into rows of cols + pad."""
    size = torch.exp(0.5 * torch.randn(cols + pad, generator=g, device=DEV)) * unit
    x = torch.empty(rows, cols + pad, device=DEV, dtype=TYPES[dtype])
    step = max(1, (1 << 27) // (cols + pad))
    for i in range(0, rows, step):
        part = x[i:i + step]
        part.copy_(torch.randn(part.shape, generator=g, device=DEV).mul_(size))
    return x[:, :cols]


def _four_bits(x):
    """(q, scales): x's rows in 4 bits, two values to a byte, and their scales."""
    rows, cols = x.shape
    padded = -(-cols // 128) * 128
    wide = torch.zeros(rows, padded, device=DEV)
    wide[:, :cols] = x
    blocks = wide.view(rows, padded // 32, 32)
    s = _exponents(blocks)
    v = blocks * _power(127 - s)
    a = _on_grid(v.abs())
    code = torch.where(a < 2, 2 * a, torch.where(a < 4, 2 + a, 4 + a / 2)).to(torch.uint8)
    code |= (v < 0).to(torch.uint8) << 3
    code = code.view(rows, padded)
    scales = torch.zeros(rows, -(-cols // 512) * 16, dtype=torch.uint8, device=DEV)
    scales[:, :padded // 32] = s.view(rows, -1)
    return (code[:, 0::2] | code[:, 1::2] << 4).contiguous(), scales


def prepare(case, seed):
    g = _gen(seed)
    kind = case["kind"]
    s = dict(case=case)
    if kind in ("norm", "grad"):
        rows, cols, pad = case["rows"], case["cols"], case["pad"]
        s["f"] = _hidden(rows, cols, case["dtype"], g, pad)
        if case["residual"]:
            s["x"] = _hidden(rows, cols, case["stream"], g, pad)
        if case["gate"] != "none":
            s["u"] = _hidden(rows, cols, case["dtype"], g, pad)
        for side in ("post", "pre"):
            if case[side]:
                s[side + "_weight"] = 1 + 0.2 * torch.randn(cols, generator=g, device=DEV)
                if case[side] == "layer":
                    s[side + "_bias"] = 0.2 * torch.randn(cols, generator=g, device=DEV)
        if kind == "grad":
            s["dy"] = _hidden(rows, cols, case["stream"], g, pad)
            if case["pre"]:
                s["dh"] = _hidden(rows, cols, case["dtype"], g, pad)
    elif kind == "round":
        s["x"] = _hidden(case["rows"], case["cols"], case["dtype"], g, case["pad"])
    else:
        s["b"], s["b_scales"] = _four_bits(_hidden(case["n"], case["k"], "f32", g,
                                                   unit=case["k"] ** -0.5))
        if kind == "linear":
            s["x"] = _hidden(case["m"], case["k"], case["dtype"], g, case["pad"])
        else:
            s["a"], s["a_scales"] = _four_bits(_hidden(case["m"], case["k"], "f32", g))
        if case["bias"]:
            s["bias"] = torch.randn(case["n"], generator=g, device=DEV)
    if own:
        _prepare_own(s)
    return s


def _prepare_own(s):
    """The output buffers and workspaces that a caller keeps, and the call's other arguments."""
    import paper_2609_22441_amd as P
    case, kind = s["case"], s["case"]["kind"]
    if kind in ("norm", "grad"):
        rows, cols, pad = case["rows"], case["cols"], case["pad"]
        norms = {"none": P.CC_NORM_NONE, "rms": P.CC_NORM_RMS, "layer": P.CC_NORM_LAYER}
        gates = {"linear": P.CC_GATE_LINEAR, "sigmoid": P.CC_GATE_SIGMOID}
        s["how"] = how = dict(x=s.get("x"), gate=s.get("u"), scale=case["scale"])
        if case["gate"] != "none":
            how["gate_kind"] = gates[case["gate"]]
        for side in ("post", "pre"):
            if case[side]:
                how.update({side + "_norm": norms[case[side]], side + "_eps": EPS,
                            side + "_weight": s[side + "_weight"],
                            side + "_bias": s.get(side + "_bias")})
        if kind == "norm":
            s["y"] = _empty(rows, cols, case["stream"], pad)
            if case["pre"]:
                s["h"] = how["h"] = _empty(rows, cols, case["dtype"], pad)
            return
        s["df"] = _empty(rows, cols, case["dtype"], pad)
        if case["residual"]:
            s["dx"] = _empty(rows, cols, case["stream"], pad)
        if case["gate"] != "none":
            s["du"] = _empty(rows, cols, case["dtype"], pad)
        for side in ("post", "pre"):
            for what in ("weight", "bias"):
                if f"{side}_{what}" in s:
                    s[f"d_{side}_{what}"] = how[f"d_{side}_{what}"] = torch.empty(cols, device=DEV)
        how.update(dy=s["dy"], dh=s.get("dh"), dx=s.get("dx"), dgate=s.get("du"))
        size = P.cc_block_norm_grad_workspace_bytes(rows, cols)
        s["workspace"] = torch.empty(size, dtype=torch.uint8, device=DEV)
    elif kind == "round":
        padded = -(-case["cols"] // 128) * 128
        s["q"] = torch.empty(case["rows"], padded // 2, dtype=torch.uint8, device=DEV)
        s["scales"] = torch.empty(case["rows"], -(-case["cols"] // 512) * 16, dtype=torch.uint8,
                                  device=DEV)
        s["out"] = _empty(case["rows"], case["cols"], case["dtype"], case["pad"])
    else:
        s["out"] = _empty(case["m"], case["n"], case["dtype"])
        size = (P.cc_linear_mxfp4_workspace_bytes if kind == "linear" else
                P.cc_matmul_mxfp4_workspace_bytes)(case["m"], case["n"], case["k"])
        s["workspace"] = torch.empty(size, dtype=torch.uint8, device=DEV)


# ---- one pass ----

def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(s):
    import paper_2609_22441_amd as P
    case, kind = s["case"], s["case"]["kind"]
    if kind == "norm":
        P.cc_block_norm(s["f"], s["y"], **s["how"])
        return _named(s, "y", "h")
    if kind == "grad":
        P.cc_block_norm_grad(s["f"], s["df"], s["workspace"], **s["how"])
        return _named(s, *GRADIENTS)
    out = s["out"]
    if kind == "round":
        P.cc_quantize_mxfp4(s["x"], s["q"], s["scales"])
        P.cc_dequantize_mxfp4(s["q"], s["scales"], out)
    elif kind == "linear":
        P.cc_linear_mxfp4(s["x"], s["b"], s["b_scales"], out, bias=s.get("bias"), relu=case["relu"],
                          workspace=s["workspace"])
    else:
        P.cc_matmul_mxfp4(s["a"], s["a_scales"], s["b"], s["b_scales"], out, bias=s.get("bias"),
                          relu=case["relu"], workspace=s["workspace"])
    return out


GRADIENTS = ("dx", "df", "du", "d_post_weight", "d_post_bias", "d_pre_weight", "d_pre_bias")


def _named(values, *names):
    return {name: values[name] for name in names if values.get(name) is not None}


def _unit(v, norm):
    """(v normalised, 1 / its size) of rows."""
    if norm == "layer":
        v = v - v.mean(1, keepdim=True)
    if norm == "none":
        return v, torch.ones_like(v[:, :1])
    r = torch.rsqrt((v * v).mean(1, keepdim=True) + EPS)
    return v * r, r


def _affine(v, s, side):
    v = v * s[side + "_weight"]
    return v + s[side + "_bias"] if side + "_bias" in s else v


def _gate(s):
    """(g, its derivative) or numbers."""
    if "u" not in s:
        return 1.0, 0.0
    u = s["u"].float()
    if s["case"]["gate"] == "linear":
        return u, 1.0
    g = 1 / (1 + torch.exp(-u))
    return g, g * (1 - g)


def _back(t, unit, r, norm):
    """The gradient of a norm's input from that of its normalised rows."""
    if norm == "none":
        return t
    d = t - unit * (t * unit).mean(1, keepdim=True)
    if norm == "layer":
        d = d - t.mean(1, keepdim=True)
    return d * r


def _run_plain(s):
    case, kind = s["case"], s["case"]["kind"]
    if kind in ("norm", "grad"):
        unit, r = _unit(s["f"].float(), case["post"])
        n = _affine(unit, s, "post")
        g, dg = _gate(s)
        y = case["scale"] * g * n
        if case["residual"]:
            y = s["x"].float() + y
        if case["pre"]:
            yunit, yr = _unit(y, case["pre"])
        dtype, stream = TYPES[case["dtype"]], TYPES[case["stream"]]
        if kind == "norm":
            out = dict(y=y.to(stream))
            if case["pre"]:
                out["h"] = _affine(yunit, s, "pre").to(dtype)
            return out
        out = {}
        dy = s["dy"].float()
        if case["pre"]:
            dh = s["dh"].float()
            dy = dy + _back(dh * s["pre_weight"], yunit, yr, case["pre"])
            out["d_pre_weight"] = (dh * yunit).sum(0)
            if "pre_bias" in s:
                out["d_pre_bias"] = dh.sum(0)
        if case["residual"]:
            out["dx"] = dy.to(stream)
        t = dy * case["scale"]
        if "u" in s:
            out["du"] = (t * n * dg).to(dtype)
        t = t * g
        out["d_post_weight"] = (t * unit).sum(0)
        if "post_bias" in s:
            out["d_post_bias"] = t.sum(0)
        out["df"] = _back(t * s["post_weight"], unit, r, case["post"]).to(dtype)
        return _named(out, *GRADIENTS)
    if kind == "round":
        return _rounded(s["x"].float()).to(TYPES[case["dtype"]])
    a = _rounded(s["x"].float()) if kind == "linear" else \
        _values(s["a"], s["a_scales"])[:, :case["k"]]
    y = a @ _values(s["b"], s["b_scales"])[:, :case["k"]].t()
    if case["bias"]:
        y = y + s["bias"]
    if case["relu"]:
        y = torch.clamp(y, min=0)
    return y.to(TYPES[case["dtype"]])


def _power(e):
    """2^e in 32 bits, for e in [-126, 127]."""
    return ((e + 127) << 23).to(torch.int32).view(torch.float32)


def _exponents(blocks):
    """The scales' biased exponents of [rows, blocks, 32], as [rows, blocks, 1] integers."""
    most = blocks.abs().amax(2, keepdim=True)
    return (((most.view(torch.int32) + (1 << 21)) >> 23) - 2).clamp(min=0)


def _on_grid(a):
    """Magnitudes rounded to the grid: steps of 0.5 up to 2, of 1 up to 4, of 2 up to 6."""
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    return torch.clamp(torch.round(a / step) * step, max=6.0)


def _rounded(x):
    """The values that the 4-bit form of x stands for."""
    rows, cols = x.shape
    wide = x
    if cols % 32:
        wide = torch.zeros(rows, -(-cols // 32) * 32, device=DEV)
        wide[:, :cols] = x
    blocks = wide.reshape(rows, -1, 32)
    s = _exponents(blocks)
    v = blocks * _power(127 - s)
    v = torch.where(v < 0, -1.0, 1.0) * _on_grid(v.abs()) * _power(s - 127)
    return v.view(rows, -1)[:, :cols]


def _values(q, scales):
    """The values of a 4-bit matrix in 32 bits."""
    code = torch.stack([q & 15, q >> 4], 2).view(q.shape[0], -1).int()
    grid = torch.tensor(GRID + tuple(-v for v in GRID), device=DEV)
    power = _power(scales[:, :q.shape[1] // 16].int() - 127)
    v = grid[code].view(q.shape[0], -1, 32) * power[:, :, None]
    return v.view(q.shape[0], -1)


# ---- what a pass cannot do without ----

def work(case):
    kind = case["kind"]
    if kind in ("norm", "grad"):
        each, stream = SIZE[case["dtype"]], SIZE[case["stream"]]
        gate, pre, res = case["gate"] != "none", case["pre"] != "", case["residual"]
        if kind == "norm":
            per = each * (1 + gate + pre) + stream * (res + 1)          # f, u, h; x, y
        else:
            # f, u, dh, df, du; x (for the second norm), dy, dx
            per = each * (2 + 2 * gate + pre) + stream * ((res and pre) + 1 + res)
        vectors = sum((1 + (case[side] == "layer")) for side in ("post", "pre") if case[side])
        elements = case["rows"] * case["cols"]
        return {"bytes": elements * per + 4 * vectors * case["cols"] * (1 + (kind == "grad")),
                "flops": elements * (20 if kind == "norm" else 50)}
    if kind == "round":
        elements = case["rows"] * case["cols"]
        return {"bytes": elements * (2 * SIZE[case["dtype"]] + 2 * 17 / 32), "flops": 4 * elements}
    m, n, k = case["m"], case["n"], case["k"]
    rows = m * k * (SIZE[case["dtype"]] if kind == "linear" else 17 / 32)
    return {"bytes": rows + n * k * 17 / 32 + (4 * n if case["bias"] else 0) +
            m * n * SIZE[case["dtype"]], "flops": 2 * m * n * k}


# ---- the definitions in 64 bits ----

def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind in ("norm", "grad"):
        return _exact_norm(case, s)
    if kind == "round":
        return torch.cat([_exact_four_bits(x) for x in s["x"].split(_rows_at_once(case["cols"]))])
    k = case["k"]
    weights = _exact_values(s["b"], s["b_scales"], k).t()
    parts = []
    for i in range(0, case["m"], 4_096):
        a = _exact_four_bits(s["x"][i:i + 4_096]) if kind == "linear" else \
            _exact_values(s["a"][i:i + 4_096], s["a_scales"][i:i + 4_096], k)
        parts.append(torch.matmul(a, weights))
    y = torch.cat(parts)
    if case["bias"]:
        y += s["bias"].double()
    return y.relu_() if case["relu"] else y


def _rows_at_once(cols):
    return max(1, (1 << 25) // cols)


def _exact_four_bits(x):
    """Each value's nearest of the eight magnitudes, found among the midpoints between them."""
    rows, cols = x.shape
    wide = torch.nn.functional.pad(x.double(), (0, -cols % 32)).view(rows, -1, 32)
    mantissa, exponent = torch.frexp(wide.abs().max(dim=2, keepdim=True).values)
    # The largest is mantissa * 2^exponent with a mantissa from 1/2 on; from 7/8 on it rounds up.
    e = torch.where(mantissa >= 0.875, exponent, exponent - 1) - 2
    unit = torch.ldexp(torch.ones_like(mantissa), e.clamp(min=-127))
    v = wide / unit
    middle = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], device=DEV, dtype=torch.float64)
    a = v.abs().contiguous()
    below, above = torch.bucketize(a, middle), torch.bucketize(a, middle, right=True)
    index = torch.where(below % 2 == 0, below, above)          # a midpoint goes to the even neighbour
    grid = torch.tensor(GRID, device=DEV, dtype=torch.float64)
    return (torch.copysign(grid[index], v) * unit).view(rows, -1)[:, :cols]


def _exact_values(q, scales, k):
    pairs = torch.empty(*q.shape, 2, device=DEV, dtype=torch.float64)
    for half, nibble in enumerate((q % 16, q // 16)):
        magnitude = nibble % 8
        low = magnitude.double() / 2
        # From 1 on: (1 + mantissa / 2) * 2^(exponent - 1).
        high = (1 + 0.5 * (magnitude % 2).double()) * torch.pow(2.0, (magnitude // 2).double() - 1)
        value = torch.where(magnitude < 2, low, high)
        pairs[..., half] = torch.where(nibble >= 8, -value, value)
    v = pairs.view(q.shape[0], -1)
    units = torch.pow(2.0, scales.double() - 127).repeat_interleave(32, dim=1)
    return (v * units[:, :v.shape[1]])[:, :k]


def _exact_norm(case, s):
    rows, cols = case["rows"], case["cols"]
    both = case["pre"] != ""
    weight = {n: s[n].double() if n in s else None
              for n in ("post_weight", "post_bias", "pre_weight", "pre_bias")}
    done, sums = {}, {}

    def centred(v, norm):
        """(centred rows, their size): the normalised rows are the quotient."""
        if norm == "none":
            return v, torch.ones(v.shape[0], 1, device=DEV, dtype=torch.float64)
        if norm == "layer":
            v = v - v.sum(1, keepdim=True) / cols
        return v, torch.sqrt(v.square().sum(1, keepdim=True) / cols + EPS)

    def norm_grad(d, v, size, norm):
        """d / size less its parts along the rows (and, centred, along ones)."""
        if norm == "none":
            return d
        along = (d * v).sum(1, keepdim=True) / cols / size.pow(3)
        out = d / size - v * along
        return out - d.sum(1, keepdim=True) / cols / size if norm == "layer" else out

    def add(name, v):
        sums[name] = sums.get(name, 0) + v.sum(0)

    def put(name, v):
        done.setdefault(name, []).append(v)

    step = _rows_at_once(cols)
    for i in range(0, rows, step):
        part = {n: s[n][i:i + step].double() for n in ("f", "x", "u", "dy", "dh") if n in s}
        v, size = centred(part["f"], case["post"])
        n = v / size * weight["post_weight"]
        if weight["post_bias"] is not None:
            n = n + weight["post_bias"]
        g, slope = torch.ones((), device=DEV, dtype=torch.float64), None
        if case["gate"] == "linear":
            g, slope = part["u"], torch.ones((), device=DEV, dtype=torch.float64)
        elif case["gate"] == "sigmoid":
            g = torch.sigmoid(part["u"])
            slope = g * torch.sigmoid(-part["u"])
        y = n * g * case["scale"]
        if case["residual"]:
            y = y + part["x"]
        if both:
            z, ysize = centred(y, case["pre"])
        if case["kind"] == "norm":
            put("y", y)
            if both:
                h = z / ysize * weight["pre_weight"]
                put("h", h + weight["pre_bias"] if weight["pre_bias"] is not None else h)
            continue
        dy = part["dy"]
        if both:
            dy = dy + norm_grad(part["dh"] * weight["pre_weight"], z, ysize, case["pre"])
            add("d_pre_weight", part["dh"] * z / ysize)
            if weight["pre_bias"] is not None:
                add("d_pre_bias", part["dh"])
        if case["residual"]:
            put("dx", dy)
        dn = dy * g * case["scale"]
        if slope is not None:
            put("du", dy * n * slope * case["scale"])
        add("d_post_weight", dn * v / size)
        if weight["post_bias"] is not None:
            add("d_post_bias", dn)
        put("df", norm_grad(dn * weight["post_weight"], v, size, case["post"]))
    out = {n: torch.cat(v) for n, v in done.items()}
    out.update(sums)
    return {n: out[n] for n in ("y", "h") + GRADIENTS if n in out}
