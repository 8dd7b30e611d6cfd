"""Layer operators at the edges of their tiles, launches and buffers (see test_gpu_layers.py for the operators themselves)."""
import pytest
import torch

from paper_1901_08227_b200 import tng
from test_gpu_layers import random_codes

pytestmark = pytest.mark.gpu


def wanted(a, sa, b, sb, dtype):
    return ((a.double() @ b.double().t()).round().float() * sa[:, None] * sb[None, :]).to(dtype)


# Split contractions whose last tile leaves warps, half a pair or most of a tile outside the matrix: those take no part in the
# exchange of sums, and nobody leaves before the others have read theirs.  (rows, columns, contraction)
SPLITS = [(1, 2503, 4096), (9, 2503, 4096), (9, 33, 8192), (17, 129, 4096), (40, 1, 4096), (33, 161, 8192), (64, 2503, 2048), (64, 96, 8192),
          (65, 2503, 4096), (100, 257, 4096), (128, 16, 8192), (129, 513, 2048), (200, 33, 4096), (300, 1, 4096), (513, 290, 4096)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("m,n,k", SPLITS)
def test_split_contractions_with_parts_outside_the_matrix(dtype, m, n, k):
    a, sa = random_codes(m, k, m + k)
    b, sb = random_codes(n, k, n + k)
    c, sc = random_codes(m, k, m + k + 1)
    want, other = wanted(a, sa, b, sb, dtype), wanted(c, sc, b, sb, dtype)
    outs = [torch.full((m, n), float("nan"), dtype=dtype, device="cuda") for _ in range(40)]
    for i, out in enumerate(outs):                          # back to back: the next launch's CTAs come in as these leave
        tng.product8(*((a, sa) if i % 2 == 0 else (c, sc)), b, sb, out=out)
    assert all(torch.equal(out, other if i % 2 else want) for i, out in enumerate(outs))


@pytest.mark.parametrize("m,n,k", [(512, 512, 64), (2600, 5000, 48), (300, 20000, 16)])
def test_whole_tiles_back_to_back(m, n, k):
    """Tiles of one block of the contraction: a pair's last hand-backs come right before it leaves."""
    a, sa = random_codes(m, k, 1)
    b, sb = random_codes(n, k, 2)
    want = wanted(a, sa, b, sb, torch.bfloat16)
    outs = [torch.full((m, n), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(10)]
    for out in outs:
        tng.product8(a, sa, b, sb, out=out)
    assert all(torch.equal(out, want) for out in outs)


@pytest.mark.parametrize("make,shape", [(tng.quant8_rows, (1, 1001)), (tng.quant8_cols, (1001, 1))])
def test_codes_of_one_line_leave_what_follows_alone(make, shape):
    pool = torch.full((2048,), 7, dtype=torch.int8, device="cuda")
    x = torch.randn(shape, device="cuda")
    with pytest.raises(ValueError):
        make(x, q=pool[:1001].view(1, 1001))
    make(x, q=pool.as_strided((1, 1001), (1008, 1)))
    assert not pool[1001:1008].any() and bool((pool[1008:] == 7).all())
