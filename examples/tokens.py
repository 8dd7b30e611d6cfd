"""A small token model trained by M workers whose gradients are exchanged as TNG codes, its matrices updated orthogonally.

    x = table[ids] sqrt(width);  u = x + relu(norm(x) W1^T) W2^T;  logits = norm(u) head^T

The norms hand their rows to the 8-bit products as codes, every worker's gradients (the table's and the norms' among them) are
written straight into its row of `grads`, one `Context.step` codes, averages and decodes the rows, and the aggregate's two inner
matrices become orthogonal updates before they are applied.  Data: each token is followed by a fixed other one.

    python examples/tokens.py [steps]
"""
from __future__ import annotations

import sys
from pathlib import Path

import torch

if __package__ in (None, ""):
    sys.path.insert(0, str(Path(__file__).resolve().parent.parent))
from paper_1901_08227_b200 import tng  # noqa: E402


class TokenModel:
    """Parameters live in one float32 vector, gradients in one row of the same layout."""

    def __init__(self, vocab, width, hidden, seed, device="cuda"):
        self.vocab, self.width, self.hidden = vocab, width, hidden
        self.shapes = [(vocab, width), (width,), (hidden, width), (width, hidden), (width,), (vocab, width)]
        self.d = sum(torch.Size(s).numel() for s in self.shapes)
        self.scale = width ** 0.5
        g = torch.Generator(device=device)
        g.manual_seed(seed)
        self.vector = torch.zeros(self.d, device=device)
        self.table, self.n1, self.w1, self.w2, self.n2, self.head = self.parts(self.vector)
        self.n1.fill_(1.0)
        self.n2.fill_(1.0)
        for w in (self.table, self.w1, self.w2, self.head):
            w.copy_(torch.randn(w.shape, generator=g, device=device) * w.shape[1] ** -0.5)

    def parts(self, row):
        """Views of a parameter-sized row as (table, n1, w1, w2, n2, head)."""
        views, at = [], 0
        for shape in self.shapes:
            n = torch.Size(shape).numel()
            views.append(row[at:at + n].view(shape))
            at += n
        return views

    def code_weights(self):
        """8-bit codes of the matrices, by row for the forward products and by column for the gradients: once a step."""
        self.rows = [tng.quant8_rows(w) for w in (self.w1, self.w2, self.head)]
        self.cols = [tng.quant8_cols(w) for w in (self.w1, self.w2, self.head)]

    def forward(self, ids, dtype=torch.bfloat16, training=True):
        """Logits (float32) and what the backward pass needs; a single token is fine."""
        x = tng.embed(self.table, ids, scale=self.scale, dtype=dtype)
        y1, y2 = (torch.empty_like(x), torch.empty_like(x)) if training else (None, None)
        q, s, _, r1 = tng.rmsnorm8(x, self.n1, y=y1)
        a = tng.product8(q, s, *self.rows[0], dtype=dtype)
        h = torch.relu(a)
        z = tng.linear8(h, *self.rows[1])
        q, s, u, r2 = tng.rmsnorm8(z, self.n2, residual=x, y=y2)
        return tng.product8(q, s, *self.rows[2], dtype=torch.float32), (ids, x, y1, r1, a, h, u, y2, r2)

    def backward(self, dlogits, saved, row):
        """Gradients of the parameters into `row`."""
        ids, x, y1, r1, a, h, u, y2, r2 = saved
        table, n1, w1, w2, n2, head = self.parts(row)
        dy2, _, _ = tng.linear8_grad(dlogits.to(x.dtype), y2, *self.cols[2], dw=head)
        du, _ = tng.rmsnorm_grad(dy2, u, self.n2, r2, dw=n2)
        dh, _, _ = tng.linear8_grad(du, h, *self.cols[1], dw=w2)
        dy1, _, _ = tng.linear8_grad(dh * (a > 0), y1, *self.cols[0], dw=w1)
        dx, _ = tng.rmsnorm_grad(dy1, x, self.n1, r1, dres=du, dw=n1)
        tng.embed_grad(dx, ids, self.vocab, scale=self.scale, dtable=table)

    def update(self, aggregate, rate, matrix_rate):
        """The two inner matrices by their orthogonalised aggregate, everything else along the aggregate itself."""
        for w in self.parts(aggregate)[2:4]:
            v = tng.orthogonalize(w)
            w.copy_(v * (matrix_rate / rate * max(1.0, w.shape[0] / w.shape[1]) ** 0.5))
        tng.sgd_update(self.vector, aggregate, rate)


def train(steps=60, workers=4, tokens=512, vocab=1000, width=256, hidden=512, rate=2.0, matrix_rate=0.02, seed=0):
    model = TokenModel(vocab, width, hidden, seed + 1)
    ld = (model.d + 3) // 4 * 4
    ctx = tng.Context(model.d, workers, 4, tng.CODEC_QSGD4, tng.NORM_DIFF, block=256, seed_lo=seed)
    grads = torch.zeros((workers, ld), device="cuda")
    out = torch.empty(model.d, device="cuda")
    g = torch.Generator(device="cuda")
    g.manual_seed(seed + 2)
    losses = []
    for _ in range(steps):
        model.code_weights()
        loss = 0.0
        for m in range(workers):
            ids = (torch.rand(tokens, generator=g, device="cuda").square() * vocab).long().clamp(max=vocab - 1)
            target = (ids * 7 + 3) % vocab
            logits, saved = model.forward(ids)
            p = torch.softmax(logits, 1)
            loss -= p.gather(1, target[:, None]).clamp_min(1e-30).log().mean().item() / workers
            p.scatter_add_(1, target[:, None], torch.full((tokens, 1), -1.0, device="cuda"))
            model.backward(p / tokens, saved, grads[m])
        ctx.step(grads, out)
        model.update(out, rate, matrix_rate)
        losses.append(loss)
    ctx.close()
    return losses


if __name__ == "__main__":
    n = int(sys.argv[1]) if len(sys.argv) > 1 else 60
    for i, v in enumerate(train(n)):
        if i % 10 == 0 or i == n - 1:
            print(f"step {i:4d}  loss {v:.5f}")
