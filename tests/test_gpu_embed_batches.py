"""The gradient of the embedding for training batches: more than 8192 tokens into tables of at least 1024 elements a token, whose zeros
take longer than the sort (four CTAs sort there; eight where the table is smaller).

A sum of n values in fp32, in any order, is off by at most n u times the sum of their magnitudes, u = 2^-24, the product with the scale by u
more (to first order; 1.01 covers the rest for n < 2^17)."""
import pytest
import torch

from paper_1901_08227_b200 import tng

pytestmark = pytest.mark.gpu
DTYPES = [torch.float32, torch.bfloat16, torch.float16]
U = 2.0 ** -24


def normal(shape, dtype, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda").to(dtype)


def ids_of(tokens, vocab, seed):
    """Falling off like 1 / rank, with empty places."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    ids = ((vocab + 1.0) ** torch.rand(tokens, generator=g, device="cuda", dtype=torch.float64) - 1).long().clamp(0, vocab - 1)
    ids[torch.rand(tokens, generator=g, device="cuda") < 0.05] = -1
    return ids


def check(dy, ids, vocab, scale, got):
    live = (ids >= 0) & (ids < vocab)
    at = torch.where(live, ids.long(), vocab)
    want = torch.zeros((vocab + 1, dy.shape[1]), dtype=torch.float64, device="cuda").index_add_(0, at, dy.double())
    size = torch.zeros_like(want).index_add_(0, at, dy.double().abs())
    count = torch.zeros(vocab + 1, dtype=torch.float64, device="cuda").index_add_(0, at, torch.ones_like(at, dtype=torch.float64))
    bad = ~((got.double() - want[:-1] * scale).abs() <= (1.01 * abs(scale) * U * (count[:, None] + 2) * size)[:-1])
    assert not bool(bad.any()), f"{int(bad.sum())} of {bad.numel()} off"


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("tokens,vocab,width", [(8193, 8200, 1024), (9000, 30000, 400), (16384, 65536, 512), (20001, 262144, 96), (12345, 262143, 65), (8300, 131, 66560),
                                                (8200, 4200000, 3), (65536, 131072, 520)])
def test_training_batches(dtype, tokens, vocab, width):
    assert tokens > 8192 and tokens * 1024 <= vocab * width
    dy, ids = normal((tokens, width), dtype, width), ids_of(tokens, vocab, tokens + vocab)
    got = tng.embed_grad(dy, ids, vocab, scale=0.37)
    check(dy, ids, vocab, 0.37, got)
    assert torch.equal(tng.embed_grad(dy, ids.to(torch.int32), vocab, scale=0.37), got)          # and the same bits each time


@pytest.mark.parametrize("tokens", [8193, 20000])
@pytest.mark.parametrize("kind", ["one id", "two ids", "all empty", "sorted", "reversed", "each once", "outside"])
def test_extreme_training_batches(tokens, kind):
    vocab, width = 30000, 700
    assert tokens > 8192 and tokens * 1024 <= vocab * width
    t = torch.arange(tokens, device="cuda")
    ids = {"one id": t * 0 + 17, "two ids": (t % 2) * (vocab - 1), "all empty": t * 0 - 1, "sorted": t // 3, "reversed": (tokens - 1 - t) // 40,
           "each once": t * 7919 % vocab, "outside": torch.where(t % 3 == 0, t, vocab + t)}[kind]
    dy = normal((tokens, width), torch.float32, tokens)
    check(dy, ids, vocab, 1.0, tng.embed_grad(dy, ids, vocab))


@pytest.mark.parametrize("lead,pad", [(0, 8), (1, 0), (3, 5)])
def test_a_training_batch_into_a_part_of_a_row(lead, pad):
    vocab, width, tokens = 20001, 516, 9001
    assert tokens > 8192 and tokens * 1024 <= vocab * width
    ld = width + pad
    buf = torch.full((lead + vocab * ld + 3,), 7.0, device="cuda")
    d = buf.as_strided((vocab, width), (ld, 1), lead)
    dy, ids = normal((tokens, width), torch.bfloat16, 3), ids_of(tokens, vocab, 4)
    tng.embed_grad(dy, ids, vocab, dtable=d)
    check(dy, ids, vocab, 1.0, d)
    d.fill_(7.0)
    assert bool((buf == 7).all())


def test_a_captured_training_batch_replays_on_new_inputs():
    vocab, width, tokens = 30000, 400, 9000
    dy, ids = normal((tokens, width), torch.bfloat16, 3), ids_of(tokens, vocab, 4)
    tng.embed_grad(dy, ids, vocab)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = tng.embed_grad(dy, ids, vocab)
    for seed in (7, 8):
        ids.copy_(ids_of(tokens, vocab, seed))
        dy.copy_(normal((tokens, width), torch.bfloat16, seed))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, tng.embed_grad(dy, ids, vocab))
