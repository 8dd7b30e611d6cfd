"""The training-layer operators together, as the feed-forward example uses them."""
import importlib.util
from pathlib import Path

import pytest
import torch

from paper_1901_08227_b200 import tng

pytestmark = pytest.mark.gpu


def example():
    path = Path(__file__).resolve().parent.parent / "examples" / "feedforward.py"
    spec = importlib.util.spec_from_file_location("feedforward", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("dtype,tokens", [(torch.float32, 200), (torch.bfloat16, 137)])
def test_gradients_are_those_of_the_block_up_to_coding(dtype, tokens):
    """Against autograd in 64 bits with the same dropout mask and the same pattern of active units (a pre-activation near
    zero may get the other sign by coding, which no bound on the products covers).  A factor coded to 8 bits is off by uniform noise of
    (max/127)/sqrt(12) an element, 1% of its rms for normal values (max about 4.5 rms; stochastic rounding: twice the
    variance); a product of two coded factors by about 2%, a chain of up to four by less than 6% in norm."""
    ff = example()
    block = ff.FeedForward(96, 160, 5)
    block.code_weights()
    x = torch.randn(tokens, 96, device="cuda").to(dtype)
    dy = torch.randn(tokens, 96, device="cuda").to(dtype)
    draw = tng.Draw(11, layer=2, step=3)
    row = torch.full((block.d,), float("nan"), device="cuda")
    y, saved = block.forward(x, draw)
    dx = block.backward(dy, saved, draw, row)
    assert bool(torch.isfinite(row).all())
    mask = tng.dropout(torch.ones_like(x), block.p, draw).double()
    v = block.vector.double().requires_grad_()
    x64 = x.double().requires_grad_()
    w1, b1, w2, b2 = block.parts(v)
    active = (saved[1] > 0).double()
    y64 = x64 + mask * ((active * (x64 @ w1.t() + b1)) @ w2.t() + b2)
    y64.backward(dy.double())
    for got, want in ((y, y64.detach()), (row, v.grad), (dx, x64.grad)):
        assert ((got.double() - want).norm() / want.norm()).item() < 0.06
    for got, want in zip(block.parts(row.double()), block.parts(v.grad)):
        assert ((got - want).norm() / want.norm()).item() < 0.06


def test_workers_train_the_block_and_the_loss_falls():
    losses = example().train(steps=40, workers=4, tokens=128, width=128, hidden=256, lr=2.0)
    assert losses[-1] < 0.5 * losses[0]


def test_serving_one_token_equals_its_row_of_a_batch():
    ff = example()
    block = ff.FeedForward(512, 768 + 16, 1)
    block.code_weights()
    x = torch.randn(200, 512, device="cuda").to(torch.bfloat16)
    whole, _ = block.forward(x, None)
    for rows in (slice(0, 1), slice(7, 15), slice(30, 60), slice(100, 200)):
        part, _ = block.forward(x[rows], None)
        assert torch.equal(part, whole[rows])                  # every kernel variant gives the same bits
