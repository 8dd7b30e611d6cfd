"""Norms and their gradients over batches in which a team of threads has several rows, against 64-bit definitions on the GPU.

Rows of more than 1024 columns that start and end on 16-byte boundaries come by bulk copies from 297 rows up; a block has teams of one or
more warps, each with up to four rows under way.  The row counts below leave the teams one to nine rows each, so that their last rows end in
every place.

Bounds.  u = 2^-24 is half a step of fp32, half(t) = finfo(t).eps / 2 that of the outputs' type.  A sum of n products in fp32, in
any order, is off by at most (n + 1) u times the sum of their magnitudes (to first order; 1.01 covers the rest for n < 2^17)."""
import pytest
import torch

from paper_1901_08227_b200 import tng

pytestmark = pytest.mark.gpu
DTYPES = [torch.float32, torch.bfloat16, torch.float16]
U = 2.0 ** -24


def half(dtype):
    return torch.finfo(dtype).eps / 2


def normal(shape, dtype, seed, scale=1.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


def close(got, want, bound):
    got, want = got.double(), want.double()
    bad = ~((got - want).abs() <= bound)
    assert not bool(bad.any()), f"{int(bad.sum())} of {bad.numel()} off, worst {((got - want).abs() / bound.clamp(min=1e-300))[bad].max().item():.3g} bounds"


def grad_check(dy, h, w, r, dres, dx, dw):
    k, n = dy.shape[1], dy.shape[0]
    d, h64, r64, w64 = dy.double(), h.double(), r.double()[:, None], w.double()
    g = d * w64
    dot, size = (g * h64).sum(1, keepdim=True), (g * h64).abs().sum(1, keepdim=True)
    along = h64 * r64 ** 2 / k
    want = r64 * (g - along * dot)
    # the sum of k products of a product each, r r dot / k: four roundings; g, the fused product, the product with r: three
    err = r64 * (along.abs() * size * (k + 7) * 1.01 * U + g.abs() * 3.03 * U + (along * dot).abs() * 3.03 * U)
    if dres is not None:
        want = want + dres.double()
        err = err + U * 1.01 * want.abs()
    close(dx, want, err + half(dx.dtype) * (want.abs() + err) + torch.finfo(dx.dtype).smallest_normal * half(dx.dtype))
    terms = d * h64 * r64
    close(dw, terms.sum(0), 1.01 * (n + 2) * U * terms.abs().sum(0))


def dx_alone(dy, h, w, r, dres):
    """dx by the C call that is given no dw."""
    (rows, cols), dx, P = dy.shape, torch.empty_like(dy), lambda t: None if t is None else t.data_ptr()
    status = tng.lib().tng_rmsnorm_grad(P(dy), cols, P(h), cols, tng._DTYPE[dy.dtype], rows, cols, P(w), P(r), P(dres), cols, P(dx), cols, None, None,
                                        torch.cuda.current_stream().cuda_stream)
    assert status == tng.OK
    return dx


def norm_check(x, w, eps, residual, y, q, scale, h, r):
    """h as stored, r and y in 64 bits; codes and their scale before r by fp32 steps."""
    k = x.shape[1]
    want_h = x if residual is None else (x.float() + residual.float()).to(x.dtype)
    h64 = want_h.double()
    want_r = 1.0 / (h64.square().mean(1) + eps).sqrt()
    want_y = h64 * want_r[:, None] * w.double()
    want_q, want_s = tng.quant8_rows(want_h.float() * w)    # (tested on its own)
    assert torch.equal(h, want_h) and torch.equal(q, want_q)
    rel = 1.01 * (k / 2 + 4) * U                            # the mean's sum, division, sum with eps: halved by the root; its rounding
    close(r, want_r, rel * want_r)
    # two products and the type's rounding (a step of its smallest number below that)
    close(y, want_y, ((rel + 2.02 * U) * (1 + half(y.dtype)) + half(y.dtype)) * want_y.abs() + torch.finfo(y.dtype).smallest_normal * half(y.dtype))
    close(scale, want_s.double() * want_r, (rel + 1.01 * U) * want_s.double() * want_r)


BATCHES = [(300, 1028), (500, 1032), (1500, 1536), (300, 2048), (701, 2048), (500, 4096), (1500, 4096), (4096, 4096), (449, 8192), (1301, 8192), (600, 11264), (600, 16384)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols", BATCHES + [(3000, 1032), (2500, 3000), (3001, 6016)])
def test_norm(dtype, rows, cols):
    x, residual, w = normal((rows, cols), dtype, cols), normal((rows, cols), dtype, cols + 1, 3.0), 1 + normal((cols,), torch.float32, 5, 0.1)
    for res in (None, residual):
        y8 = torch.empty_like(x)
        q, s, h, r = tng.rmsnorm8(x, w, residual=res, y=y8)
        norm_check(x, w, 1e-6, res, y8, q, s, h, r)
        y, h2, r2 = tng.rmsnorm(x, w, residual=res)
        assert torch.equal(y, y8) and torch.equal(h2, h) and torch.equal(r2, r)
        for into in ("x", "residual"):
            if into == "x" or res is not None:
                a, b = x.clone(), None if res is None else res.clone()
                q3, s3, h3, r3 = tng.rmsnorm8(a, w, residual=b, h=None if res is None else a if into == "x" else b)
                assert torch.equal(h3, h) and torch.equal(r3, r) and torch.equal(q3, q) and torch.equal(s3, s)
        a = x.clone()
        assert torch.equal(tng.rmsnorm(a, w, residual=res, y=a)[0], y)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols", BATCHES)
def test_norm_grad(dtype, rows, cols):
    h, w = normal((rows, cols), dtype, 1, 2.0), 1 + normal((cols,), torch.float32, 5, 0.1)
    dy, res = normal((rows, cols), dtype, 2, 0.1), normal((rows, cols), dtype, 3, 0.1)
    r = torch.rsqrt(h.float().square().mean(1) + 1e-6)
    for dres in (None, res):
        dx, dw = tng.rmsnorm_grad(dy, h, w, r, dres=dres)
        grad_check(dy, h, w, r, dres, dx, dw)
        assert torch.equal(dx_alone(dy, h, w, r, dres), dx)
        for into in ("dy", "dres"):
            if into == "dy" or dres is not None:
                a, b = dy.clone(), None if dres is None else dres.clone()
                again = tng.rmsnorm_grad(a, h, w, r, dres=b, dx=a if into == "dy" else b)
                assert torch.equal(again[0], dx) and torch.equal(again[1], dw)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols", [(1, 16400), (70, 16385), (200, 20000), (3, 100003)])
def test_norm_grad_in_place_of_rows_longer_than_a_block_holds(dtype, rows, cols):
    """dx and dw are two kernels there, and either reads dy."""
    h, w = normal((rows, cols), dtype, 1, 2.0), 1 + normal((cols,), torch.float32, 5, 0.1)
    dy, res = normal((rows, cols), dtype, 2, 0.1), normal((rows, cols), dtype, 3, 0.1)
    r = torch.rsqrt(h.float().square().mean(1) + 1e-6)
    for dres, into in ((None, "dy"), (res, "dy"), (res, "dres")):
        a, b = dy.clone(), None if dres is None else dres.clone()
        dx, dw = tng.rmsnorm_grad(a, h, w, r, dres=b, dx=a if into == "dy" else b)
        grad_check(dy, h, w, r, dres, dx, dw)
