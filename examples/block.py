"""A block of the scoring model on hidden rows: training steps, then serving with weights in 4 bits
(W h + b with ReLU, the norms after and before a block, its gate and the residual sum: Connected Content
Retriever, §4, Eq. 2).

    python examples/block.py

A block reads h, the norm of the residual stream x, and gives f = ReLU(W h + b); the stream goes on as
x + scale * sigmoid(u) * norm(f), and h for the next block is the norm of that. Training keeps x, f and
the gate u of a block and computes its norms again in the backward pass. Serving writes y over x and h
over f, with W in microscaled 4-bit floating point.
"""
from __future__ import annotations

import sys
from pathlib import Path

sys.path.insert(0, str(Path(__file__).resolve().parents[1]))

import torch  # noqa: E402

import paper_2609_22441_amd as P  # noqa: E402

SCALE = 0.5


class Block:
    """W, b of the layer, U of its gate, and the weights of the norms around it."""

    def __init__(self, cols, device, seed=1):
        g = torch.Generator(device=device).manual_seed(seed)
        self.w = torch.randn(cols, cols, generator=g, device=device) / cols ** 0.5
        self.u = torch.randn(cols, cols, generator=g, device=device) / cols ** 0.5
        self.b = torch.zeros(cols, device=device)
        self.post = torch.ones(cols, device=device)
        self.pre = torch.ones(cols, device=device)

    def norms(self):
        return dict(scale=SCALE, post_norm=P.CC_NORM_LAYER, post_weight=self.post, post_eps=1e-5,
                    pre_norm=P.CC_NORM_RMS, pre_weight=self.pre, pre_eps=1e-6)

    def layer(self, h):
        """f and the gate in bf16 from h."""
        return torch.relu(h.float() @ self.w.t() + self.b).bfloat16(), (h.float() @ self.u.t()).bfloat16()

    def forward(self, x, h):
        f, gate = self.layer(h)
        y, next_h = torch.empty_like(x), torch.empty_like(h)
        P.cc_block_norm(f, y, x=x, gate=gate, h=next_h, **self.norms())
        return f, gate, y, next_h

    def backward(self, x, h, f, gate, dh, dy=None):
        """Gradients of x, of h, and of the block's parameters from those of the next h and of y."""
        n, cols = f.shape
        df, dgate, dx = torch.empty_like(f), torch.empty_like(gate), torch.empty_like(x)
        grads = {k: torch.empty_like(self.post) for k in ("d_post_weight", "d_pre_weight")}
        work = torch.empty(P.cc_block_norm_grad_workspace_bytes(n, cols), dtype=torch.uint8,
                           device=f.device)
        P.cc_block_norm_grad(f, df, work, x=x, gate=gate, dy=dy, dh=dh, dx=dx, dgate=dgate, **grads,
                             **self.norms())
        df = df.float() * (f > 0)
        return dx, df @ self.w + dgate.float() @ self.u, dict(
            w=df.t() @ h.float(), u=dgate.float().t() @ h.float(), b=df.sum(0),
            post=grads["d_post_weight"], pre=grads["d_pre_weight"])


class Serving:
    """The same block with W and U in 4 bits."""

    def __init__(self, block):
        self.block = block
        self.w, self.u = (self.four_bits(x) for x in (block.w, block.u))

    @staticmethod
    def four_bits(w):
        rows, cols = w.shape
        q = torch.empty(rows, -(-cols // 128) * 64, dtype=torch.uint8, device=w.device)
        scales = torch.empty(rows, -(-cols // 512) * 16, dtype=torch.uint8, device=w.device)
        P.cc_quantize_mxfp4(w, q, scales)
        return q, scales

    def __call__(self, x, h):
        """y over x, and the next block's h."""
        m, cols = h.shape
        work = torch.empty(P.cc_linear_mxfp4_workspace_bytes(m, cols, cols), dtype=torch.uint8,
                           device=h.device)
        f, gate = torch.empty_like(h), torch.empty_like(h)
        P.cc_linear_mxfp4(h, *self.w, f, bias=self.block.b, relu=True, workspace=work)
        P.cc_linear_mxfp4(h, *self.u, gate, workspace=work)
        P.cc_block_norm(f, x, x=x, gate=gate, h=f, **self.block.norms())
        return x, f


def hidden(rows, cols, device, seed=2):
    """(the residual stream, its norm in bf16)."""
    g = torch.Generator(device=device).manual_seed(seed)
    x = torch.randn(rows, cols, generator=g, device=device)
    return x, (x / x.square().mean(1, keepdim=True).sqrt()).bfloat16()


def main():
    device = torch.device("cuda:0")
    x, h = hidden(4_000, 512, device)
    block = Block(512, device)
    target = torch.roll(h.float(), 1, dims=1)
    for number in range(8):
        f, gate, _, out = block.forward(x, h)
        error = out.float() - target
        dh = (error * (2 / error.shape[0])).bfloat16()
        *_, grads = block.backward(x, h, f, gate, dh)
        for name, g in grads.items():
            getattr(block, name).sub_(0.05 * g)
        print(f"step {number}: loss {float(error.square().sum(1).mean()):.4f}", flush=True)
    *_, y, out = block.forward(x, h)
    served, served_h = Serving(block)(x.clone(), h)
    error = (served_h.float() - out.float()).norm() / out.float().norm()
    print(f"serving: {tuple(served.shape)}, {float(error):.4f} from the block in 32 bits", flush=True)


if __name__ == "__main__":
    main()
