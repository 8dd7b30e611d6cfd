"""A residual feed-forward block trained by M workers whose gradients are exchanged as TNG codes.

    y = x + dropout(relu(x W1^T + b1) W2^T + b2)

The block's matrix products run in 8-bit integers (forward and gradients), dropout recomputes its mask in the backward
pass, every worker's weight gradients are written straight into its row of `grads`, and one `Context.step` codes,
averages and decodes the rows.  Data: a fixed random block of the same shape is the teacher.

    python examples/feedforward.py [steps]
"""
from __future__ import annotations

import sys
from pathlib import Path

import torch

if __package__ in (None, ""):
    sys.path.insert(0, str(Path(__file__).resolve().parent.parent))
from paper_1901_08227_b200 import tng  # noqa: E402


class FeedForward:
    """Parameters live in one float32 vector, gradients in one row of the same layout."""

    def __init__(self, width, hidden, seed, p=0.1, device="cuda"):
        self.width, self.hidden, self.p = width, hidden, p
        shapes = [(hidden, width), (hidden,), (width, hidden), (width,)]
        self.d = sum(torch.Size(s).numel() for s in shapes)
        g = torch.Generator(device=device)
        g.manual_seed(seed)
        self.vector = torch.zeros(self.d, device=device)
        self.w1, self.b1, self.w2, self.b2 = self.parts(self.vector)
        self.w1.copy_(torch.randn(hidden, width, generator=g, device=device) * width ** -0.5)
        self.w2.copy_(torch.randn(width, hidden, generator=g, device=device) * hidden ** -0.5)

    def parts(self, row):
        """Views of a parameter-sized row as (w1, b1, w2, b2)."""
        h, n = self.hidden, self.width
        a, b, c = h * n, h * n + h, 2 * h * n + h
        return row[:a].view(h, n), row[a:b], row[b:c].view(n, h), row[c:c + n]

    def code_weights(self):
        """8-bit codes of both matrices, by row for the forward products and by column for dx: once a step."""
        self.q1, self.s1 = tng.quant8_rows(self.w1)
        self.q2, self.s2 = tng.quant8_rows(self.w2)
        self.t1, self.u1 = tng.quant8_cols(self.w1)
        self.t2, self.u2 = tng.quant8_cols(self.w2)

    def forward(self, x, draw):
        """draw = None: no dropout (serving; a single token is fine)."""
        a = tng.linear8(x, self.q1, self.s1, bias=self.b1.contiguous())
        h = torch.relu(a)
        z = tng.linear8(h, self.q2, self.s2, bias=self.b2.contiguous())
        y = x + z if draw is None else tng.dropout(z, self.p, draw, residual=x)
        return y, (x, a, h)

    def backward(self, dy, saved, draw, row):
        """Gradients of the parameters into `row`; returns the gradient of x."""
        x, a, h = saved
        w1, b1, w2, b2 = self.parts(row)
        rounding = tng.Draw(draw.seed_lo | draw.seed_hi << 32, draw.layer + 1, draw.step, draw.row0)
        dz = tng.dropout_grad(dy, self.p, draw)
        dh, _, _ = tng.linear8_grad(dz, h, self.t2, self.u2, draw=draw, dw=w2, db=b2)
        da = dh * (a > 0)
        dx, _, _ = tng.linear8_grad(da, x, self.t1, self.u1, draw=rounding, dw=w1, db=b1)
        return dy + dx


def train(steps=60, workers=4, tokens=256, width=256, hidden=512, lr=2.0, seed=0, dtype=torch.bfloat16):
    teacher = FeedForward(width, hidden, seed + 1, p=0.0)
    teacher.code_weights()
    block = FeedForward(width, hidden, seed + 2)
    ld = (block.d + 3) // 4 * 4
    ctx = tng.Context(block.d, workers, 4, tng.CODEC_QSGD4, tng.NORM_DIFF, block=256, seed_lo=seed)
    grads = torch.zeros((workers, ld), device="cuda")
    out = torch.empty(block.d, device="cuda")
    g = torch.Generator(device="cuda")
    g.manual_seed(seed + 3)
    x = torch.randn((workers * tokens, width), generator=g, device="cuda").to(dtype)
    target, _ = teacher.forward(x, None)
    losses = []
    for t in range(steps):
        block.code_weights()
        loss = 0.0
        for m in range(workers):
            rows = slice(m * tokens, (m + 1) * tokens)
            draw = tng.Draw(seed, layer=0, step=t, row0=m * tokens)   # a worker draws what the whole batch would
            y, saved = block.forward(x[rows], draw)
            err = y.float() - target[rows].float()
            loss += err.square().mean().item() / workers
            block.backward((2.0 / err.numel() * err).to(dtype), saved, draw, grads[m])
        ctx.step(grads, out)
        tng.sgd_update(block.vector, out, lr)
        losses.append(loss)
    ctx.close()
    return losses


if __name__ == "__main__":
    n = int(sys.argv[1]) if len(sys.argv) > 1 else 60
    for i, v in enumerate(train(n)):
        if i % 10 == 0 or i == n - 1:
            print(f"step {i:4d}  loss {v:.5f}")
