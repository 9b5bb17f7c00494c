"""Learned rows and a dense layer on joined rows: training steps of a position table, then serving in 8-bit
integers (dropout and ReLU(W h + b): Connected Content Retriever, §4, Eq. 2).

    python examples/input_layer.py

Both start from the join: every candidate's document row and its viewer's edge row for the document's
author, 96 bf16 columns. Training adds a row for the candidate's slot, number min(slot, S_max) of a table, to
the rows under dropout, and learns the table by the gradient that cc_embedding_grad sums by slot. (This is
the example's own use of a table of rows. The paper's Eq. 3 adds a slot's row to the model's 3 logits: the
same two calls with a table of 3 columns.) Serving adds the learned rows and runs the first dense layer,
ReLU(W h + b), in 8-bit integers.
"""
from __future__ import annotations

import sys
from pathlib import Path

sys.path.insert(0, str(Path(__file__).resolve().parents[1]))

import torch  # noqa: E402

import paper_2609_22441_amd as P  # noqa: E402
import workload as W  # noqa: E402

S_MAX = 50                    # later slots share the last row of the table
P_DROP = 0.1


def joined_rows(device, viewers=4, candidates=2_000, seed=1):
    """[viewers * candidates, 96] bf16 rows and each candidate's row of the position table."""
    spec, req = W.shape(2, store_n_docs=50_000, store_n_authors=50_000, req_n_viewers=viewers,
                        req_n_cand=candidates, req_k=1_000)
    data = W.make_store(spec, seed, device="cpu")
    batch = W.pack(W.make_requests(data, req, seed)).to(device)
    store = P.cc_store_create(data.author_id.to(device), data.doc_rows.to(device))
    total = batch.cand_idx.numel()
    rows = torch.empty(total, spec.doc_cols + req.edge_cols, dtype=torch.bfloat16, device=device)
    hit = torch.empty(total, dtype=torch.int8, device=device)
    P.cc_join_batched(store, batch.cand_offsets, batch.cand_idx, batch.key_offsets, batch.keys,
                      batch.edge_rows, rows, hit)
    torch.cuda.synchronize()
    P.cc_store_destroy(store)
    slots = torch.arange(candidates, device=device).clamp_(max=S_MAX).repeat(viewers)
    return rows, slots


class Training:
    """A position table under plain gradient descent; the head's weights are fixed."""

    def __init__(self, rows, slots, seed=7):
        g = torch.Generator(device=rows.device).manual_seed(seed)
        n, cols = rows.shape
        self.rows, self.slots, self.seed = rows, slots, seed
        self.table = torch.zeros(S_MAX + 1, cols, device=rows.device)
        self.head = torch.randn(cols, generator=g, device=rows.device) / cols ** 0.5
        self.target = rows.float() @ self.head + torch.cos(slots / 8.0)      # a bias by position
        self.pos, self.hidden = torch.empty_like(rows), torch.empty_like(rows)
        self.grad = torch.empty_like(self.table)
        self.workspace = torch.empty(P.cc_embedding_grad_workspace_bytes(n, S_MAX + 1, cols),
                                     dtype=torch.uint8, device=rows.device)

    def step(self, number, rate=0.5):
        """One step; the masks of a step follow from its number, and the backward pass draws the
        lookup's again. Returns the loss before the update."""
        seed = self.seed << 32 | number
        P.cc_embedding_lookup(self.table, self.slots, self.pos, p=P_DROP, seed=seed, site=0)
        P.cc_dropout(self.rows, self.hidden, P_DROP, seed, site=1, residual=self.pos)
        error = self.hidden.float() @ self.head - self.target
        d_hidden = (error[:, None] * self.head).to(torch.bfloat16)
        P.cc_embedding_grad(self.slots, d_hidden, self.grad, self.workspace, p=P_DROP, seed=seed,
                            site=0)
        count = torch.bincount(self.slots, minlength=S_MAX + 1)[:, None]
        self.table -= rate * self.grad / count
        return error.square().mean()


class Serving:
    """rows + table[slots] -> ReLU(W h + b) with W quantised once."""

    def __init__(self, table, weights, bias):
        outputs, cols = weights.shape
        self.table, self.bias = table, bias
        self.w = torch.empty(outputs, -(-cols // 16) * 16, dtype=torch.int8, device=weights.device)
        self.w_scales = torch.empty(outputs, device=weights.device)
        P.cc_quantize_rows(weights, self.w, self.w_scales)

    def __call__(self, rows, slots):
        m, cols = rows.shape
        hidden = torch.empty_like(rows)
        P.cc_embedding_lookup(self.table, slots, hidden)
        hidden += rows
        out = torch.empty(m, self.w.shape[0], dtype=rows.dtype, device=rows.device)
        workspace = torch.empty(P.cc_linear_i8_workspace_bytes(m, self.w.shape[0], cols),
                                dtype=torch.uint8, device=rows.device)
        P.cc_linear_i8(hidden, self.w, self.w_scales, out, bias=self.bias, relu=True,
                       workspace=workspace)
        return out


def main():
    device = torch.device("cuda:0")
    rows, slots = joined_rows(device)
    training = Training(rows, slots)
    for number in range(8):
        print(f"step {number}: loss {float(training.step(number)):.4f}", flush=True)
    g = torch.Generator(device=device).manual_seed(3)
    weights = torch.randn(512, rows.shape[1], generator=g, device=device) / rows.shape[1] ** 0.5
    bias = torch.randn(512, generator=g, device=device)
    out = Serving(training.table, weights, bias)(rows, slots)
    plain = torch.relu((rows + training.table[slots].bfloat16()).float() @ weights.t() + bias)
    error = (out.float() - plain).norm() / plain.norm()
    print(f"serving: {tuple(out.shape)}, {float(error):.4f} from the product in 32 bits", flush=True)


if __name__ == "__main__":
    main()
