"""The operators of a token model together, as the example uses them."""
import importlib.util
import math
from pathlib import Path

import pytest
import torch

from paper_1901_08227_b200 import tng

pytestmark = pytest.mark.gpu


def example():
    path = Path(__file__).resolve().parent.parent / "examples" / "tokens.py"
    spec = importlib.util.spec_from_file_location("tokens", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def norm64(x, w):
    return x / (x.square().mean(1, keepdim=True) + 1e-6).sqrt() * w


@pytest.mark.parametrize("dtype,tokens", [(torch.float32, 200), (torch.bfloat16, 333)])
def test_gradients_are_those_of_the_model_up_to_coding(dtype, tokens):
    """Against autograd in 64 bits with the same pattern of active units.  A product of two factors coded to 8 bits is off by about 2% in
    norm (uniform noise of max / 127 / sqrt(12) an element, 1% of the rms of normal values, on either side); no gradient passes more than
    five such products one after another (both matrices forward, the head and both matrices backward): 10% if all of it adds up."""
    ex = example()
    model = ex.TokenModel(300, 96, 160, 5)
    model.code_weights()
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    ids = torch.randint(0, 300, (tokens,), generator=g, device="cuda")
    ids[::17] = -1                                          # padding
    dlogits = torch.randn((tokens, 300), generator=g, device="cuda")
    dlogits[ids < 0] = 0                                    # and nothing is learnt from it
    row = torch.full((model.d,), float("nan"), device="cuda")
    logits, saved = model.forward(ids, dtype)
    model.backward(dlogits, saved, row)
    assert bool(torch.isfinite(row).all())
    v = model.vector.double().requires_grad_()
    table, n1, w1, w2, n2, head = model.parts(v)
    live = (ids >= 0)[:, None]
    x = torch.where(live, table[ids.clamp(min=0)] * model.scale, torch.zeros((), dtype=torch.float64, device="cuda"))
    active = (saved[4] > 0).double()
    u = x + (active * (norm64(x, n1) @ w1.t())) @ w2.t()
    want = norm64(u, n2) @ head.t()
    assert ((logits.double() - want)[live[:, 0]].norm() / want[live[:, 0]].norm()).item() < 0.1
    want.backward(dlogits.double())
    for got, ref in zip(model.parts(row.double()), model.parts(v.grad)):
        assert ((got - ref).norm() / ref.norm()).item() < 0.1
    named = torch.zeros(300, dtype=torch.bool, device="cuda")
    named[ids[ids >= 0]] = True
    assert not model.parts(row)[0][~named].any()            # rows of the table that no token names


def test_serving_one_token_equals_its_row_of_a_batch():
    ex = example()
    model = ex.TokenModel(1000, 512, 768 + 16, 1)
    model.code_weights()
    ids = torch.randint(0, 1000, (200,), device="cuda")
    whole, _ = model.forward(ids, training=False)
    for rows in (slice(0, 1), slice(7, 15), slice(30, 63), slice(100, 200)):
        part, _ = model.forward(ids[rows], training=False)
        # the same codes in every variant; the scales hold a sum of 512 squares whose order depends on the rows' number: (512 / 2 + 4) 2^-24
        # each for two norms, the second of rows that may differ in their last bit of bf16 (2^-8) and then in a code or two
        assert ((part - whole[rows]).norm() / whole[rows].norm()).item() < 2.0 ** -8


def test_workers_train_the_model():
    losses = example().train(steps=6, workers=3, tokens=130, vocab=257, width=64, hidden=96)
    assert len(losses) == 6 and all(math.isfinite(v) for v in losses)


def test_an_update_moves_the_matrices_orthogonally():
    ex = example()
    model = ex.TokenModel(50, 96, 160, 5)
    before = model.vector.clone()
    aggregate = torch.randn(model.d, device="cuda")
    want = aggregate.clone()
    model.update(aggregate, rate=0.5, matrix_rate=0.02)
    moved = model.parts(before - model.vector)
    for i, (got, v) in enumerate(zip(moved, model.parts(want))):
        if i not in (2, 3):
            assert torch.allclose(got, 0.5 * v, atol=1e-6, rtol=1e-5)
        else:                                               # singular values within the polynomial's range around one, times the rate
            s = torch.linalg.svdvals(got.double()) / (0.02 * max(1.0, v.shape[0] / v.shape[1]) ** 0.5)
            assert s.max().item() < 1.21 and s.min().item() > 0.3
