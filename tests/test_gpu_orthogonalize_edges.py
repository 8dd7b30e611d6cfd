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


MUON = (3.4445, -4.7750, 2.0315)


def fp32_form(v, steps, coefficients=MUON):
    """Elementary fp32 operations throughout."""
    a, b, c = coefficients
    x = v.float()
    tall = x.shape[0] > x.shape[1]
    x = x.t() if tall else x
    x = x / torch.sqrt(x.double().square().sum()).float()
    for _ in range(steps):
        g = x @ x.t()
        x = a * x + (b * g + c * (g @ g)) @ x
    return x.t() if tall else x


def aggregate(m, n, seed):
    """A few strong directions over noise, as an aggregate has."""
    rank = max(1, min(m, n) // 16)
    fall = torch.exp(-4.0 * torch.arange(rank, device="cuda") / rank)
    return 1e-3 * normal((m, n), seed=seed) + 1e-2 * (normal((m, rank), seed=seed + 1) * fall) @ normal((rank, n), seed=seed + 2) / rank ** 0.5


@pytest.mark.parametrize("kind", [normal, aggregate])
@pytest.mark.parametrize("m,n", [(512, 512), (515, 1001), (1001, 515), (640, 640), (1024, 1024), (2048, 2304), (1024, 4096)])
def test_the_error_is_of_the_order_of_fp32_products(kind, m, n):
    """Five steps, as fp32: at most twice the error that fp32 products have on the same matrix.  (Sums left to the matrix unit over four or
    eight blocks of the contraction would have two and a half times that and five times.)"""
    v = normal((m, n), seed=m + n) if kind is normal else aggregate(m, n, m + n)
    want = wanted(v, 5)
    own, plain = ((f.double() - want).norm().item() for f in (tng.orthogonalize(v), fp32_form(v, 5)))
    assert own < 2 * plain


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("kind", [normal, aggregate])
@pytest.mark.parametrize("m,n", [(1024, 4096), (1100, 4200), (4100, 1030)])
def test_several_steps_at_once_before_their_rounding(dtype, kind, m, n):
    """Results in 16 bits whose sides differ twofold take several steps with one Gram matrix.  What they are off by before the rounding to the
    type: an entry that is off by d rounds to the neighbour of what the exact one rounds to in one of (step / d) cases, and is then a step off, so
    that the mean distance from the rounded exact entries is the mean of |d| (over millions of entries within a few percent).  Two to four
    times the error of fp32 products is what products of 22-bit factors leave; factors of 11 bits, a half lost on the way, would leave 2^-12."""
    v = normal((m, n), seed=m + n) if kind is normal else aggregate(m, n, m + n)
    want = wanted(v, 5)
    off = (tng.orthogonalize(v, dtype=dtype).double() - want.to(dtype).double()).abs().sum().item()
    assert off < 4 * (fp32_form(v, 5).double() - want).abs().sum().item()


@pytest.mark.parametrize("shrink", [1e-2, 1e-4, 1e-6, 1e-8])
@pytest.mark.parametrize("m,n,side", [(256, 512, 0), (256, 512, 1), (512, 256, 0), (512, 256, 1), (1030, 2100, 0)])
def test_rows_and_columns_that_are_much_smaller_than_the_rest(m, n, side, shrink):
    """Factors are held with fixed steps: half of one is 2^-39 for X, 2^-38 for G, 2^-37 for B.  With s and l the sides and singular values of at most
    1.21, a step adds at most e = 2^-39 (14.8 sqrt(l) + 23.6 sqrt(s)) to the error of a line of X, whatever its size: a sqrt(l) from X itself,
    1.21 (b + 1.46 c) (1.21 sqrt(l) + 2 sqrt(s)) by way of G, 1.21 * 4 sqrt(s) by way of B; later steps let it grow a-fold each.  The rest is
    relative: one step's share at most 2^-19 of the line, which grows likewise."""
    v = normal((m, n), seed=m)
    small = v[:32] if side == 0 else v[:, :32]
    small *= shrink
    want, got = wanted(v, 5), tng.orthogonalize(v).double()
    s, l = min(m, n), max(m, n)
    grown = sum(3.4445 ** k for k in range(5))
    step = 2.0 ** -39 * (14.8 * l ** 0.5 + 23.6 * s ** 0.5)
    error, size = ((t[:32] if side == 0 else t[:, :32].t()).norm(dim=1) for t in (got - want, want))
    assert bool((error < grown * (step + 2.0 ** -19 * size)).all())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("kind", [normal, aggregate])
@pytest.mark.parametrize("m,n", [(512, 512), (640, 512), (515, 1001)])
def test_small_16_bit_results_differ_from_the_rounded_exact_ones_at_ties_alone(dtype, kind, m, n):
    """Step by step: before the rounding to the type the error is that of the fp32 result (its mean as above; ties met are few here, about
    one entry in a thousand, so a third more is allowed for chance), and an entry is one step off at most."""
    v = normal((m, n), seed=m + n) if kind is normal else aggregate(m, n, m + n)
    want, got = wanted(v, 5), tng.orthogonalize(v, dtype=dtype).double()
    full = (tng.orthogonalize(v).double() - want).abs()
    off = (got - want.to(dtype).double()).abs()
    # half a step of the type (of its smallest numbers below that), and the error, which the fp32 result shows, twice
    assert bool(((got - want).abs() <= torch.finfo(dtype).eps / 2 * want.abs() + torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps + 2 * full.max()).all())
    assert off.sum().item() < 1.33 * full.sum().item()
