"""The orthogonalised update at its edges: sides beyond what one dimension of a grid counts."""
import pytest
import torch

from paper_1901_08227_b200 import tng

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def normal(shape, dtype=torch.float32, seed=1, scale=1.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


def wanted(v, steps, coefficients=(3.4445, -4.7750, 2.0315)):
    a, b, c = (float(torch.tensor(t)) for t in coefficients)
    x = v.double()
    tall = x.shape[0] > x.shape[1]
    x = x.t() if tall else x
    x = x / torch.linalg.vector_norm(x)
    for _ in range(steps):
        g = x @ x.t()
        x = a * x + (b * g + c * (g @ g)) @ x
    return x.t() if tall else x


@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("m,n", [(4194305, 3), (3, 4194305), (4500001, 8)])
def test_more_rows_than_a_grid_counts_blocks_of(m, n, out):
    """One step.  The entries are about 2^-12 and smaller.  A sum over K products in blocks of 64 is off by (K / 64 + 25) u and 3 * 2^-22 of its
    magnitudes at most, here K = 2^22 for G; what is seen of that in B X is at most b of the entry, and c twice: 2 c + b < 9 times."""
    v = normal((m, n), seed=m % 1000 + n)
    got = tng.orthogonalize(v, steps=1, dtype=out).double()
    want = wanted(v, 1)
    k = max(m, n)
    assert ((got - want).norm() / want.norm()).item() < 9 * ((k / 64 + 25) * U + 3 * 2.0 ** -22) + torch.finfo(out).eps / 2
    rows = torch.tensor([0, 63, 64, 65535 * 64 - 1, 65535 * 64, k - 1], device="cuda")
    side = 0 if m > n else 1
    a, b = got.index_select(side, rows), want.index_select(side, rows)
    assert ((a - b).norm() / b.norm()).item() < 9 * ((k / 64 + 25) * U + 3 * 2.0 ** -22) + torch.finfo(out).eps / 2
