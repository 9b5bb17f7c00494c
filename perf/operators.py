"""Timed cases of the scoring model's input layer: embedding lookup and its gradient, dropout from
a counter-based generator, and the 8-bit integer product, next to the join whose rows they take.

Each case is a dict of plain values. ``listed()`` names the fixed ones, ``draw(rng)`` gives more of
the same ranges, ``prepare`` makes what a caller holds before the call, ``run`` is one pass, in
elementary torch operations or, with ``own`` set, through the package's entry points; ``exact``
gives a pass's outputs in 64 bits.

Five kinds of case:
  lookup   rows of a table by id, scaled; with a dropout of the looked-up values in training
  grad     the table's gradient: rows of the output's gradient summed by id
  dropout  a mask drawn from (seed, site, row, column), with or without a residual sum; on a
           gradient the same call is the backward pass
  product  8-bit rows times 8-bit weights, a scale per row of each, bias and ReLU
  linear   the same from floating-point rows, quantised row by row within the call

Dropout's definition. Element (row, column) draws 16 bits: number column % 8 of the four 32-bit
words of Philox4x32-10 (Salmon et al., SC 2011) at counter (row mod 2^32, row / 2^32, column / 8,
site) under the 64-bit key `seed`, low half of a word first. It is kept where they are below
T = 65536 - floor(65536 p + 1/2), and scaled by 65536 / T.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False
DEV = "cuda"
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}
MAX_ELEMENTS = 1 << 28          # of a drawn case's largest array
MAX_MACS = 1 << 39              # of a drawn product
M32 = 0xFFFFFFFF


def listed():
    return [
        # A decoding step of a batch: one token each. Latency counts.
        _lookup("lookup_tokens", n=64, rows=32_000, cols=1_024, dtype="bf16"),
        # A training step's tokens against a large vocabulary, dropout on the embeddings.
        _lookup("lookup_train", n=131_072, rows=131_072, cols=4_096, dtype="bf16", p=0.1),
        # A small step in 32 bits with odd sizes: rows of the width that the join writes.
        _grad("grad_small", n=2_049, rows=1_000, cols=96, dtype="f32", grad="f32"),
        # Position table of 51 slots under a serving batch's 400,000 candidates: the last slot
        # stands for every later one and takes most of the rows.
        _grad("grad_slots", n=400_000, rows=51, cols=96, dtype="bf16", grad="f32", ids="slots"),
        # A training step's tokens, a 50,000-row vocabulary with Zipf frequencies, dropout.
        _grad("grad_vocab", n=131_072, rows=50_000, cols=2_048, dtype="bf16", grad="f32", p=0.1,
              bad=0.02),
        # One request's joined rows, odd in both directions.
        _dropout("dropout_request", rows=999, cols=97, dtype="f16", p=0.2),
        # A training step's hidden rows, added to the residual stream.
        _dropout("dropout_train", rows=131_072, cols=4_096, dtype="bf16", p=0.1, residual=True),
        # One token through a square layer: the weights' bytes and the launch count.
        _product("linear", "linear_token", m=1, n=4_096, k=4_096, dtype="bf16"),
        # A request's 50,000 joined rows of 96 columns through the first layer.
        _product("linear", "linear_request", m=50_000, n=512, k=96, dtype="bf16"),
        # A long prompt or a large batch through a wide layer.
        _product("linear", "linear_large", m=16_384, n=8_192, k=8_192, dtype="bf16"),
        # A few hundred rows, nothing a multiple of a tile, 32-bit output.
        _product("product", "product_ragged", m=333, n=1_030, k=2_055, dtype="f32"),
        # A wide layer of rows that are in 8 bits already.
        _product("product", "product_wide", m=8_192, n=16_384, k=4_096, dtype="bf16"),
    ]


def _lookup(name, n, rows, cols, dtype, out=None, p=0.0, ids="zipf", narrow=False, bad=0.0, pad=0,
            first=0):
    return dict(name=name, kind="lookup", n=n, rows=rows, cols=cols, dtype=dtype, out=out or dtype,
                p=p, ids=ids, narrow=narrow, bad=bad, pad=pad, first=first)


def _grad(name, n, rows, cols, dtype, grad, p=0.0, ids="zipf", narrow=False, bad=0.0, pad=0,
          first=0):
    return dict(name=name, kind="grad", n=n, rows=rows, cols=cols, dtype=dtype, grad=grad, p=p,
                ids=ids, narrow=narrow, bad=bad, pad=pad, first=first)


def _dropout(name, rows, cols, dtype, p, residual=False, pad=0, first=0):
    return dict(name=name, kind="dropout", rows=rows, cols=cols, dtype=dtype, p=p,
                residual=residual, pad=pad, first=first)


def _product(kind, name, m, n, k, dtype, bias=True, relu=True, pad=0):
    return dict(name=name, kind=kind, m=m, n=n, k=k, dtype=dtype, bias=bias, relu=relu, pad=pad)


def draw(rng):
    kind = rng.choice(["lookup", "grad", "dropout", "linear", "product"])
    while True:
        c = _DRAW[kind](rng)
        c.pop("name")
        if kind in ("linear", "product"):
            fits = c["m"] * c["n"] * c["k"] <= MAX_MACS and \
                max(c["m"] * c["n"], c["m"] * c["k"], c["n"] * c["k"]) <= MAX_ELEMENTS
        elif kind == "dropout":
            fits = c["rows"] * c["cols"] <= MAX_ELEMENTS
        else:
            fits = max(c["n"], c["rows"]) * c["cols"] <= MAX_ELEMENTS
        if fits:
            return c


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _cols(rng, lo=16, hi=8_192):
    """Columns: mostly multiples of 8, as models have them, some odd."""
    c = _log(rng, lo, hi)
    return c if rng.random() < 0.25 else max(8, c // 8 * 8)


def _table(rng):
    return dict(n=_log(rng, 1, 500_000), rows=_log(rng, 2, 200_000), cols=_cols(rng),
                dtype=rng.choice(["bf16", "bf16", "f16", "f32"]), p=rng.choice([0.0, 0.1, 0.25]),
                ids=rng.choice(["zipf", "zipf", "uniform", "slots"]), narrow=rng.random() < 0.3,
                bad=rng.choice([0.0, 0.02]), pad=rng.choice([0, 0, 8, 3]),
                first=rng.choice([0, 1_000_000, 5_000_000_000]))


def _draw_lookup(rng):
    c = _table(rng)
    return _lookup("", out=rng.choice(["f32", "bf16"]) if c["dtype"] == "f32" else None, **c)


def _draw_grad(rng):
    c = _table(rng)
    return _grad("", grad="f32" if rng.random() < 0.6 else c["dtype"], **c)


def _draw_dropout(rng):
    return _dropout("", rows=_log(rng, 1, 500_000), cols=_cols(rng),
                    dtype=rng.choice(["bf16", "bf16", "f16", "f32"]),
                    p=rng.choice([0.05, 0.1, 0.5]), residual=rng.random() < 0.5,
                    pad=rng.choice([0, 0, 8, 3]), first=rng.choice([0, 1_000_000, 5_000_000_000]))


def _draw_product(kind):
    def make(rng):
        return _product(kind, "", m=_log(rng, 1, 50_000), n=_cols(rng, 64, 16_384),
                        k=_cols(rng, 64, 16_384), dtype=rng.choice(["bf16", "bf16", "f16", "f32"]),
                        bias=rng.random() < 0.7, relu=rng.random() < 0.5,
                        pad=rng.choice([0, 0, 8, 3]) if kind == "linear" else 0)
    return make


_DRAW = {"lookup": _draw_lookup, "grad": _draw_grad, "dropout": _draw_dropout,
         "linear": _draw_product("linear"), "product": _draw_product("product")}


# ---- inputs ----

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 1_000_003 + 17)
    return g


def _probabilities(case):
    """Of the table's ranks, as a float64 array that sums to 1."""
    rows = case["rows"]
    if case["ids"] == "zipf":                       # token frequencies
        w = np.arange(1, rows + 1, dtype=np.float64) ** -1.1
        return w / w.sum()
    if case["ids"] == "slots":                      # min(slot, rows - 1) of 4 * rows slots
        w = np.ones(rows)
        w[-1] += 3 * rows
        return w / w.sum()
    return np.full(rows, 1.0 / rows)


def _ids(case, g):
    u = torch.rand(case["n"], generator=g, device=DEV, dtype=torch.float64)
    cdf = torch.from_numpy(np.cumsum(_probabilities(case))).to(DEV)
    ranks = torch.searchsorted(cdf, u).clamp_(max=case["rows"] - 1)
    if case["ids"] == "zipf":                       # frequent ids lie anywhere in the table
        ranks = torch.randperm(case["rows"], generator=g, device=DEV)[ranks]
    if case["bad"]:                                 # not found: -1
        ranks[torch.rand(case["n"], generator=g, device=DEV) < case["bad"]] = -1
    return ranks.to(torch.int32) if case["narrow"] else ranks


def _normal(rows, cols, dtype, g, pad=0):
    """N(0, 1) values, as a view into rows of cols + pad where pad > 0."""
    x = torch.randn(rows, cols + pad, generator=g, device=DEV, dtype=TYPES[dtype])
    return x[:, :cols]


def _empty(rows, cols, dtype, pad=0):
    return torch.empty(rows, cols + pad, device=DEV, dtype=TYPES[dtype])[:, :cols]


def _eight_bits(rows, cols, g):
    """(q, scales) of N(0, 1 / cols) rows: rows of q are padded with zeros to a multiple of 16."""
    x = torch.randn(rows, cols, generator=g, device=DEV) / math.sqrt(cols)
    scales = x.abs().amax(1) / 127.0
    q = torch.zeros(rows, -(-cols // 16) * 16, dtype=torch.int8, device=DEV)
    q[:, :cols] = torch.round(x / scales[:, None]).clamp_(-127, 127).to(torch.int8)
    return q, scales


def prepare(case, seed):
    g = _gen(seed)
    kind = case["kind"]
    s = dict(case=case)
    if kind in ("lookup", "grad", "dropout"):
        s["seed"] = (int(seed) * 0x9E3779B97F4A7C15 + 0x1234567) & ((1 << 64) - 1)
        s["site"] = 3
    if kind == "lookup":
        s["table"] = _normal(case["rows"], case["cols"], case["dtype"], g)
        s["ids"] = _ids(case, g)
        s["scale"] = math.sqrt(case["cols"])
    elif kind == "grad":
        s["dout"] = _normal(case["n"], case["cols"], case["dtype"], g, case["pad"])
        s["ids"] = _ids(case, g)
        s["scale"] = 0.5
    elif kind == "dropout":
        s["x"] = _normal(case["rows"], case["cols"], case["dtype"], g, case["pad"])
        if case["residual"]:
            s["residual"] = _normal(case["rows"], case["cols"], case["dtype"], g, case["pad"])
    else:
        s["b"], s["b_scales"] = _eight_bits(case["n"], case["k"], g)
        if kind == "linear":
            s["x"] = _normal(case["m"], case["k"], case["dtype"], g, case["pad"])
        else:
            s["a"], s["a_scales"] = _eight_bits(case["m"], case["k"], g)
            s["a_scales"] *= math.sqrt(case["k"])
        if case["bias"]:
            s["bias"] = torch.randn(case["n"], generator=g, device=DEV)
    if own:
        _prepare_own(s)
    return s


def _prepare_own(s):
    """The output buffers and workspaces that a caller keeps."""
    import paper_2609_22441_amd as P
    case, kind = s["case"], s["case"]["kind"]
    if kind == "lookup":
        s["out"] = _empty(case["n"], case["cols"], case["out"], case["pad"])
    elif kind == "grad":
        s["out"] = _empty(case["rows"], case["cols"], case["grad"])
        size = P.cc_embedding_grad_workspace_bytes(case["n"], case["rows"], case["cols"])
        s["workspace"] = torch.empty(size, dtype=torch.uint8, device=DEV)
    elif kind == "dropout":
        s["out"] = _empty(case["rows"], case["cols"], case["dtype"], case["pad"])
    else:
        s["out"] = _empty(case["m"], case["n"], case["dtype"])
        size = (P.cc_linear_i8_workspace_bytes if kind == "linear" else
                P.cc_matmul_i8_workspace_bytes)(case["m"], case["n"], case["k"])
        s["workspace"] = torch.empty(size, dtype=torch.uint8, device=DEV)


# ---- one pass ----

def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(s):
    import paper_2609_22441_amd as P
    case, kind = s["case"], s["case"]["kind"]
    out = s["out"]
    if kind == "lookup":
        P.cc_embedding_lookup(s["table"], s["ids"], out, scale=s["scale"], p=case["p"],
                              seed=s["seed"], site=s["site"], first_row=case["first"])
    elif kind == "grad":
        P.cc_embedding_grad(s["ids"], s["dout"], out, s["workspace"], scale=s["scale"],
                            p=case["p"], seed=s["seed"], site=s["site"], first_row=case["first"])
    elif kind == "dropout":
        P.cc_dropout(s["x"], out, case["p"], s["seed"], site=s["site"], first_row=case["first"],
                     residual=s.get("residual"))
    elif kind == "linear":
        P.cc_linear_i8(s["x"], s["b"], s["b_scales"], out, bias=s.get("bias"), relu=case["relu"],
                       workspace=s["workspace"])
    else:
        P.cc_matmul_i8(s["a"], s["a_scales"], s["b"], s["b_scales"], out, bias=s.get("bias"),
                       relu=case["relu"], workspace=s["workspace"])
    return out


def _threshold(p):
    return 65536 - int(math.floor(65536 * p + 0.5))


def _kept(rows, cols, s):
    """Dropout's mask [rows, cols] in 64-bit integer operations."""
    case, seed = s["case"], s["seed"]
    blocks = -(-cols // 8)
    row = torch.arange(case["first"], case["first"] + rows, device=DEV)[:, None]
    row = row.expand(rows, blocks)
    c0, c1 = row & M32, row >> 32
    c2 = torch.arange(blocks, device=DEV)[None, :].expand(rows, blocks)
    c3 = torch.full_like(c2, s["site"])
    k0, k1 = seed & M32, seed >> 32
    for _ in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57     # modulo 2^64: both halves are exact
        c0, c1, c2, c3 = ((b >> 32) & M32) ^ c1 ^ k0, b & M32, ((a >> 32) & M32) ^ c3 ^ k1, a & M32
        k0, k1 = (k0 + 0x9E3779B9) & M32, (k1 + 0xBB67AE85) & M32
    words = torch.stack([x for c in (c0, c1, c2, c3) for x in (c & 0xFFFF, c >> 16)], dim=2)
    return words.view(rows, blocks * 8)[:, :cols] < _threshold(case["p"])


def _dropped(x, s):
    """x with dropout's mask and scale applied."""
    p = s["case"]["p"]
    if p == 0:
        return x
    return torch.where(_kept(*x.shape, s), x * (65536 / _threshold(p)), 0.0)


def _run_plain(s):
    case, kind = s["case"], s["case"]["kind"]
    if kind == "lookup":
        ids = s["ids"].long()
        y = s["table"][ids.clamp(min=0)].float() * s["scale"]
        return _dropped(torch.where((ids >= 0)[:, None], y, 0.0), s).to(TYPES[case["out"]])
    if kind == "grad":
        ids = s["ids"].long()
        d = _dropped(s["dout"].float(), s) * s["scale"]
        g = torch.zeros(case["rows"] + 1, case["cols"], device=DEV)     # the last row: ids of -1
        g.index_add_(0, torch.where(ids >= 0, ids, case["rows"]), d)
        return g[:-1].to(TYPES[case["grad"]])
    if kind == "dropout":
        y = _dropped(s["x"].float(), s)
        if case["residual"]:
            y = y + s["residual"].float()
        return y.to(TYPES[case["dtype"]])
    if kind == "linear":
        x = s["x"].float()
        most = x.abs().amax(1, keepdim=True)
        a, a_scales = torch.round(x * (127.0 / most)), most[:, 0] / 127.0
    else:
        a, a_scales = s["a"][:, :case["k"]].float(), s["a_scales"]
    y = a @ s["b"][:, :case["k"]].float().t()
    y = y * a_scales[:, None] * s["b_scales"]
    if case["bias"]:
        y = y + s["bias"]
    if case["relu"]:
        y = torch.clamp(y, min=0)
    return y.to(TYPES[case["dtype"]])


# ---- what a pass cannot do without ----

def work(case):
    kind = case["kind"]
    if kind in ("lookup", "grad"):
        ids = case["n"] * (4 if case["narrow"] else 8)
        rows = case["n"] * (1 - case["bad"])
        if kind == "lookup":
            # Each distinct row of the table is read once.
            distinct = float(np.sum(-np.expm1(rows * np.log1p(-_probabilities(case) * (1 - 1e-9)))))
            moved = distinct * case["cols"] * SIZE[case["dtype"]] + \
                case["n"] * case["cols"] * SIZE[case["out"]]
        else:
            moved = rows * case["cols"] * SIZE[case["dtype"]] + \
                case["rows"] * case["cols"] * SIZE[case["grad"]]
        return {"bytes": ids + moved, "flops": 0 if kind == "lookup" else rows * case["cols"]}
    if kind == "dropout":
        return {"bytes": case["rows"] * case["cols"] * SIZE[case["dtype"]] *
                (3 if case["residual"] else 2), "flops": 0}
    m, n, k = case["m"], case["n"], case["k"]
    rows = m * k * SIZE[case["dtype"]] if kind == "linear" else m * k + 4 * m
    return {"bytes": rows + n * k + 4 * n + (4 * n if case["bias"] else 0) +
            m * n * SIZE[case["dtype"]], "flops": 2 * m * n * k}


# ---- the definitions in 64 bits ----

def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "dropout":
        y = torch.where(_kept_by_halves(case["rows"], case["cols"], s),
                        s["x"].double() * 65536 / _threshold(case["p"]), 0.0)
        return y + s["residual"].double() if case["residual"] else y
    if kind in ("lookup", "grad"):
        factor = s["scale"] * 65536 / _threshold(case["p"])
        ids = s["ids"].long()
        found = (ids >= 0)[:, None]
        kept = found
        if case["p"]:
            kept = found & _kept_by_halves(case["n"], case["cols"], s)
        if kind == "lookup":
            y = torch.where(kept, s["table"].index_select(0, ids.clamp(min=0)), 0.0)
            return y.double().mul_(factor)
        g = torch.zeros(case["rows"], case["cols"], device=DEV, dtype=torch.float64)
        step = max(1, (1 << 26) // case["cols"])
        for i in range(0, case["n"], step):
            d = torch.where(kept[i:i + step], s["dout"][i:i + step].double(), 0.0)
            g.scatter_add_(0, ids[i:i + step].clamp(min=0)[:, None].expand_as(d), d)
        return g.mul_(factor)
    b = s["b"][:, :case["k"]].double() * s["b_scales"].double()[:, None]
    if kind == "linear":
        x = s["x"].double()
        unit = x.abs().max(dim=1, keepdim=True).values / 127
        a = torch.round(x / unit).mul_(unit)
    else:
        a = s["a"][:, :case["k"]].double() * s["a_scales"].double()[:, None]
    y = torch.matmul(a, b.t())
    if case["bias"]:
        y += s["bias"].double()
    return y.relu_() if case["relu"] else y


def _kept_by_halves(rows, cols, s):
    """Dropout's mask from the generator's definition, its 64-bit products put together from
    16-bit halves, which no step takes past 2^53; the columns of one 8-column block at a time."""
    case, t = s["case"], _threshold(s["case"]["p"])

    def product(x, m):
        """(high, low) 32 bits of x * m."""
        low = (x & 0xFFFF) * m                       # below 2^48
        high = (x >> 16) * m                         # below 2^48
        mid = (low >> 16) + high                     # the product is mid * 2^16 + low % 2^16
        return mid >> 16, ((mid & 0xFFFF) << 16) | (low & 0xFFFF)

    row = torch.arange(rows, device=DEV) + case["first"]
    kept = torch.empty(rows, -(-cols // 8) * 8, dtype=torch.bool, device=DEV)
    step = max(1, (1 << 22) // max(rows, 1))         # blocks taken together
    for first in range(0, -(-cols // 8), step):
        block = torch.arange(first, min(first + step, -(-cols // 8)), device=DEV)
        word = [(row % (1 << 32))[:, None] + 0 * block, (row // (1 << 32))[:, None] + 0 * block,
                0 * row[:, None] + block, s["site"] + 0 * (row[:, None] + block)]
        for r in range(10):
            key = [((s["seed"] % (1 << 32)) + r * 0x9E3779B9) % (1 << 32),
                   ((s["seed"] // (1 << 32)) + r * 0xBB67AE85) % (1 << 32)]
            h0, l0 = product(word[0], 0xD2511F53)
            h1, l1 = product(word[2], 0xCD9E8D57)
            word = [h1 ^ word[1] ^ key[0], l1, h0 ^ word[3] ^ key[1], l0]
        for j in range(8):
            bits = (word[j // 2] >> 16) if j % 2 else word[j // 2] % (1 << 16)
            kept[:, first * 8 + j:(first + block.numel()) * 8:8] = bits < t
    return kept[:, :cols]
