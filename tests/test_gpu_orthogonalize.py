"""The orthogonalised update against 64 bits.

Bounds.  u = 2^-24.  A factor held in two fp16 halves is off by at most 2^-22 of it, and so is a product that leaves out the product of
the low halves.  The matrix unit's sum over a block of 64 takes twelve instructions, each off by at most one fp32 step (2 u) of
the magnitudes so far; blocks are added to nearest, u each.  An entry of P Q^T over K is then off by at most eta(K) times that of
|P| |Q|^T, eta(K) = 3 * 2^-22 + 24 u + (K / 64 + 1) u; one step's error follows entry by entry.  Over several steps what a step leaves
grows with the slope of the polynomial and its chords, at most a = 3.4445 for these coefficients; with one step's share at most
2^-19 of the norm, n steps stay below 2^-19 (1 + a + ... + a^(n-1)) for matrices whose norm does not shrink."""
import pytest
import torch

from paper_1901_08227_b200 import tng

pytestmark = pytest.mark.gpu
DTYPES = [torch.float32, torch.bfloat16, torch.float16]
U = 2.0 ** -24
MUON = (3.4445, -4.7750, 2.0315)
CLASSIC = (1.875, -1.25, 0.375)
CUBIC = (1.5, -0.5, 0.0)


def normal(shape, dtype=torch.float32, seed=1, scale=1.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


def eta(k):
    return 3 * 2.0 ** -22 + (24 + k / 64 + 1) * U


def wide(v):
    """v in 64 bits, shorter side first."""
    x = v.double()
    return (x.t(), True) if x.shape[0] > x.shape[1] else (x, False)


def wanted(v, steps, coefficients=MUON):
    a, b, c = (float(torch.tensor(t)) for t in coefficients)
    x, tall = wide(v)
    x = x / torch.linalg.vector_norm(x)
    for _ in range(steps):
        g = x @ x.t()
        x = a * x + (b * g + c * (g @ g)) @ x
    return x.t() if tall else x


def one_step_bound(v, coefficients=MUON):
    """Entry by entry, before the rounding to the output's type."""
    a, b, c = (abs(t) for t in coefficients)
    x, tall = wide(v)
    x = x.abs() / torch.linalg.vector_norm(x)
    s, l = x.shape
    held = 2.0 ** -22                                       # of a factor; X itself also by its division and fp32 rounding
    g = x @ x.t()
    dg = (eta(l) + 4 * U) * g + held * g
    poly = a * torch.eye(s, dtype=torch.float64, device=x.device) + b * g + c * g @ g
    db = b * dg + c * (2 * (g @ dg) + eta(s) * (g @ g)) + (held + 4 * U) * poly
    d = db @ x + (eta(s) + 4 * U) * (poly @ x)
    d = 1.01 * d + 2.0 ** -36                               # (2^-36: the low halves' smallest step, 2^-24 / 2^14, and what a product makes of it)
    return d.t() if tall else d


def rel(got, want):
    return ((got.double() - want).norm() / want.norm()).item()


def growth(steps, a=3.4445):
    return 2.0 ** -19 * sum(a ** k for k in range(steps))


SIZES = [(1, 1), (1, 300), (300, 1), (2, 3), (64, 64), (127, 129), (128, 128), (129, 127), (100, 3000), (256, 512), (257, 300), (515, 1001), (1001, 515), (640, 640),
         (31, 5000), (1500, 1300)]


@pytest.mark.parametrize("m,n", SIZES)
@pytest.mark.parametrize("coefficients", [MUON, CLASSIC, CUBIC])
def test_one_step_entry_by_entry(m, n, coefficients):
    v = normal((m, n), seed=m + n)
    got = tng.orthogonalize(v, steps=1, coefficients=coefficients)
    want = wanted(v, 1, coefficients)
    bad = (got.double() - want).abs() > one_step_bound(v, coefficients) + U * want.abs()
    assert not bool(bad.any())


@pytest.mark.parametrize("m,n", [(2304, 4100), (4100, 2304)])      # tiles of two SMs
def test_one_step_of_large_matrices(m, n):
    v = normal((m, n), seed=m)
    want = wanted(v, 1)
    assert not bool(((tng.orthogonalize(v, steps=1).double() - want).abs() > one_step_bound(v) + U * want.abs()).any())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("out", DTYPES)
@pytest.mark.parametrize("m,n", [(64, 200), (300, 129), (515, 1001)])
def test_types(dtype, out, m, n):
    v = normal((m, n), dtype, m)
    got = tng.orthogonalize(v, dtype=out)
    assert got.dtype == out and rel(got, wanted(v, 5)) < growth(5) + torch.finfo(out).eps / 2
    assert out != dtype or torch.equal(tng.orthogonalize(v), got)


@pytest.mark.parametrize("steps", [1, 2, 3, 5, 6])
@pytest.mark.parametrize("m,n", [(200, 333), (333, 200), (2048, 2304)])
def test_steps(steps, m, n):
    v = normal((m, n), seed=steps)
    assert rel(tng.orthogonalize(v, steps=steps), wanted(v, steps)) < growth(steps)


# Sides that differ twofold and 16-bit results: several steps with one Gram matrix.
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("steps", [1, 2, 3, 4, 5, 6, 7])
@pytest.mark.parametrize("m,n", [(1100, 4200), (4100, 1030)])
@pytest.mark.parametrize("coefficients", [MUON, CLASSIC])
def test_several_steps_at_once(dtype, steps, m, n, coefficients):
    v = normal((m, n), seed=steps)
    assert rel(tng.orthogonalize(v, steps=steps, coefficients=coefficients, dtype=dtype), wanted(v, steps, coefficients)) < growth(steps) + torch.finfo(dtype).eps / 2


@pytest.mark.parametrize("m,n", [(1100, 4200), (4100, 1030)])
def test_several_steps_at_once_of_a_batch(m, n):
    v = normal((3, m, n), torch.bfloat16, 4)
    got = tng.orthogonalize(v)
    assert all(rel(got[i], wanted(v[i], 5)) < growth(5) + torch.finfo(torch.bfloat16).eps / 2 for i in range(3))
    v[1, 3, 4] = float("nan")
    again = tng.orthogonalize(v)
    assert torch.equal(again[0], got[0]) and torch.equal(again[2], got[2]) and bool(again[1].isnan().all())


def test_singular_values_come_near_one():
    """The classic coefficients converge; singular values from 0.02 of the norm up are at one within 2^-10 after twelve steps."""
    g = torch.linalg.qr(normal((300, 200)).double())[0] * torch.linspace(1.0, 0.1, 200, dtype=torch.float64, device="cuda")
    v = (g @ torch.linalg.qr(normal((200, 200), seed=2).double())[0]).float()
    x = tng.orthogonalize(v, steps=12, coefficients=CLASSIC).double()
    assert (x.t() @ x - torch.eye(200, dtype=torch.float64, device="cuda")).abs().max().item() < 2.0 ** -10
    u, _, w = torch.linalg.svd(v.double(), full_matrices=False)
    assert (x - u @ w).abs().max().item() < 2.0 ** -10


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("lead,pad", [(0, 0), (0, 8), (1, 0), (3, 5)])
@pytest.mark.parametrize("m,n", [(130, 257), (257, 130)])
def test_strides_and_padding(dtype, lead, pad, m, n):
    v = normal((3, m, n), dtype, 4)
    want = tng.orthogonalize(v, dtype=torch.float32)
    for i in range(3):
        assert torch.equal(tng.orthogonalize(v[i], dtype=torch.float32), want[i])             # batched or not
    ld, gap = n + pad, m * (n + pad) + 11
    src = torch.full((lead + 3 * gap,), float("nan"), dtype=dtype, device="cuda").as_strided((3, m, n), (gap, ld, 1), lead)
    src.copy_(v)
    buf = torch.full((lead + 3 * gap,), 7.0, device="cuda")
    out = buf.as_strided((3, m, n), (gap, ld, 1), lead)
    assert tng.orthogonalize(src, out=out) is out and torch.equal(out, want)
    out.fill_(7.0)
    assert bool((buf == 7).all())
    side = torch.zeros((m, 3 * n), dtype=dtype, device="cuda")         # matrices side by side
    side.view(m, 3, n).transpose(0, 1).copy_(v)
    assert torch.equal(tng.orthogonalize(side.view(m, 3, n).transpose(0, 1), dtype=torch.float32), want)


def test_matrices_that_are_zero_or_not_finite_leave_their_neighbours_alone():
    v = normal((5, 70, 90))
    want = tng.orthogonalize(v)
    v[1] = 0
    v[2, 3, 4] = float("inf")
    v[3, 5, 6] = float("nan")
    got = tng.orthogonalize(v)
    assert torch.equal(got[0], want[0]) and torch.equal(got[4], want[4])
    assert not got[1].any() and bool(got[2:4].isnan().all())


@pytest.mark.parametrize("m,n", [(100, 140), (140, 100)])
@pytest.mark.parametrize("power", [-120, -60, 60, 120])
def test_powers_of_two_change_nothing(m, n, power):
    """Sums of squares far beyond fp32's range on either side."""
    v = normal((m, n))
    v[v.abs() < 2.0 ** -5] = 0.5                            # (nothing becomes subnormal)
    assert torch.equal(tng.orthogonalize(v * 2.0 ** power), tng.orthogonalize(v))


def test_one_strong_direction():
    """Rank one and a little noise: what is left in the weak directions is the noise's own, grown, not that of the arithmetic."""
    v = normal((200, 1)) @ normal((1, 300), seed=2) + 1e-5 * normal((200, 300), seed=3)
    want = wanted(v, 5)
    got = tng.orthogonalize(v)
    # the first step's share, 2^-19 of norm one, times 3.4445^5 in the weak directions; the result's norm is above one
    assert (got.double() - want).norm().item() < 2.0 ** -19 * sum(3.4445 ** k for k in range(6))


def test_same_bits_each_time_and_in_a_graph():
    v = normal((3, 300, 200))
    want = tng.orthogonalize(v)
    assert all(torch.equal(tng.orthogonalize(v), want) for _ in range(5))
    static, stream = v.clone(), torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        out = tng.orthogonalize(static)
    for seed in (5, 6):
        static.copy_(normal((3, 300, 200), seed=seed))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, tng.orthogonalize(static))


def test_two_streams_at_once():
    vs = [normal((700, 500), seed=i) for i in range(2)]
    want = [tng.orthogonalize(v) for v in vs]
    streams = [torch.cuda.Stream() for _ in vs]
    torch.cuda.synchronize()
    for _ in range(10):
        got = []
        for s, v in zip(streams, vs):
            with torch.cuda.stream(s):
                got.append(tng.orthogonalize(v))
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_part_of_an_aggregate():
    """A matrix of the parameter vector as a round returns it, back into the vector's place."""
    d, m, n = 100 + 96 * 160 + 60, 96, 160
    ctx = tng.Context(d, 2, 1, tng.CODEC_QSGD4, tng.NORM_DIFF, block=128)
    out = ctx.step(normal((2, d)), torch.empty(d, device="cuda"))
    part = out[100:100 + m * n].view(m, n)
    update = torch.zeros(d, device="cuda")
    tng.orthogonalize(part, out=update[100:100 + m * n].view(m, n))
    assert rel(update[100:100 + m * n].view(m, n), wanted(part, 5)) < growth(5)
    assert not update[:100].any() and not update[100 + m * n:].any()
    ctx.close()


def test_offsets_beyond_32_bits():
    ld = (1 << 30) + 64                                     # rows 4 GB apart
    buf = torch.zeros(ld + 64, device="cuda")
    far = buf.as_strided((2, 40), (ld, 1))
    near = normal((2, 40))
    far.copy_(near)
    want = tng.orthogonalize(near)
    assert torch.equal(tng.orthogonalize(far), want)
    tng.orthogonalize(near, out=far)
    assert torch.equal(far, want) and not buf[40:64].any()


def test_refusals():
    v = normal((4, 8))
    with pytest.raises(ValueError):
        tng.orthogonalize(v[0])
    with pytest.raises(ValueError):
        tng.orthogonalize(v.t())
    with pytest.raises(TypeError):
        tng.orthogonalize(v.double())
    with pytest.raises(TypeError):
        tng.orthogonalize(v.cpu())
    with pytest.raises(ValueError):
        tng.orthogonalize(v, out=torch.empty((8, 4), device="cuda"))
    with pytest.raises(TypeError):
        tng.orthogonalize(v, dtype=torch.bfloat16, out=torch.empty_like(v))
    with pytest.raises(ValueError):
        tng.orthogonalize(v, scratch=torch.empty(16, dtype=torch.uint8, device="cuda"))
    for bad in [dict(steps=0), dict(steps=65), dict(coefficients=(10.0, -9.0, 2.0)), dict(coefficients=(2.5, 0.0, 0.0)), dict(coefficients=(16.0, -60.0, 50.0)),
                dict(coefficients=(float("nan"), 0.0, 0.0)), dict(coefficients=(1.0, float("inf"), 0.0))]:
        with pytest.raises(tng.TngError) as e:
            tng.orthogonalize(v, **bad)
        assert e.value.status == tng.ERR_INVALID_ARG
    with pytest.raises(tng.TngError):
        tng.orthogonalize(normal((2, 4, 8)), out=torch.empty((1, 4, 8), device="cuda").expand(2, 4, 8))
    assert tng.orthogonalize(torch.empty((0, 4, 8), device="cuda")).shape == (0, 4, 8)
