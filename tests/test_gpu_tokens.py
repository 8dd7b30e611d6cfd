"""Embedding rows, root-mean-square norm and their gradients against 64-bit definitions on the GPU.

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


def ids_of(tokens, vocab, seed, dtype=torch.int64):
    """Falling off like 1 / rank, with empty places."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    ids = ((vocab + 1.0) ** torch.rand(tokens, generator=g, device="cuda", dtype=torch.float64) - 1).long().clamp(0, vocab - 1)
    ids[torch.rand(tokens, generator=g, device="cuda") < 0.05] = -1
    return ids.to(dtype)


def inside(rows, cols, dtype, lead, ld, fill=7.0):
    """A (rows, cols) view of a larger buffer and the buffer: rows start `lead` elements in and ld apart."""
    buf = torch.full((lead + rows * ld + 3,), fill, dtype=dtype, device="cuda")
    return buf.as_strided((rows, cols), (ld, 1), lead), buf


def untouched(buf, view, fill=7.0):
    mask = torch.ones_like(buf, dtype=torch.bool)
    mask.as_strided(view.shape, view.stride(), view.storage_offset()).fill_(False)
    return bool((buf[mask] == fill).all())


def close(got, want, bound):
    got, want = got.double(), want.double()
    bad = ~((got - want).abs() <= bound)
    assert not bool(bad.any()), f"{int(bad.sum())} of {bad.numel()} off, worst {((got - want).abs() / bound.clamp(min=1e-300))[bad].max().item():.3g} bounds"


# ---- embedding ---------------------------------------------------------------------------------------

def embed_wanted(table, ids, scale, dtype):
    y = (table[ids.long().clamp(0, table.shape[0] - 1)].float() * torch.tensor(scale, device="cuda")).to(dtype)   # one fp32 product
    y[ids == -1] = 0
    y[(ids < -1) | (ids >= table.shape[0])] = float("nan")
    return y


@pytest.mark.parametrize("table_type", DTYPES)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("tokens,vocab,width", [(1, 1, 1), (1, 100, 4096), (7, 3, 17), (300, 1000, 515), (129, 50, 1024), (64, 70, 1032), (20, 9, 9000)])
def test_embed(table_type, dtype, tokens, vocab, width):
    table, ids = normal((vocab, width), table_type, width), ids_of(tokens, vocab, tokens)
    for kind in (torch.int64, torch.int32):
        got = tng.embed(table, ids.to(kind), scale=22.6, dtype=dtype)
        assert got.dtype == dtype and torch.equal(got, embed_wanted(table, ids, 22.6, dtype))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("lead,pad", [(0, 8), (8, 16), (1, 0), (3, 5), (0, 1)])
def test_embed_rows_that_start_anywhere(dtype, lead, pad):
    width, vocab, tokens = 1000, 40, 33
    table, _ = inside(vocab, width, dtype, lead, width + pad)
    table.copy_(normal((vocab, width), dtype, 1))
    out, buf = inside(tokens, width, dtype, lead, width + pad)
    ids = ids_of(tokens, vocab, 2)
    assert tng.embed(table, ids, out=out) is out
    assert torch.equal(out, embed_wanted(table, ids, 1.0, dtype)) and untouched(buf, out)


def test_embed_ids_outside_the_table_are_nan_and_empty_places_zero():
    table = normal((10, 300), torch.float32, 1)
    for kind in (torch.int64, torch.int32):
        ids = torch.tensor([0, 9, 10, -1, -2, 2 ** 31 - 1, -2 ** 31, 5], dtype=kind, device="cuda")
        got = tng.embed(table, ids, scale=3.0)
        live = torch.tensor([0, 1, 7], device="cuda")
        assert torch.equal(got[live], table[ids[live].long()] * 3.0)
        assert not got[3].any() and bool(got[torch.tensor([2, 4, 5, 6], device="cuda")].isnan().all())
    ids = torch.tensor([2 ** 32, 2 ** 32 + 1, -2 ** 63, 2 ** 63 - 1], device="cuda")      # their low words look like rows
    assert bool(tng.embed(table, ids).isnan().all())
    assert not tng.embed_grad(normal((4, 300), torch.float32, 2), ids, 10).any()


def test_embed_of_nothing():
    table = normal((10, 30), torch.bfloat16, 1)
    none = torch.empty(0, dtype=torch.int64, device="cuda")
    assert tng.embed(table, none).shape == (0, 30)
    d = torch.full((10, 30), 5.0, device="cuda")
    tng.embed_grad(table[:0], none, 10, dtable=d)
    assert not d.any()


def embed_grad_check(dy, ids, vocab, scale, got):
    want = torch.zeros((vocab + 1, dy.shape[1]), dtype=torch.float64, device="cuda")
    live = (ids >= 0) & (ids < vocab)
    at = torch.where(live, ids.long(), vocab)
    want.index_add_(0, at, dy.double())
    size = torch.zeros_like(want).index_add_(0, at, dy.double().abs())
    count = torch.zeros(vocab + 1, dtype=torch.float64, device="cuda").index_add_(0, at, torch.ones_like(at, dtype=torch.float64))
    close(got, want[:-1] * scale, (1.01 * abs(scale) * U * (count[:, None] + 2) * size)[:-1])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("tokens,vocab,width", [(1, 1, 1), (1, 5000, 64), (31, 7, 3), (32, 1, 1000), (33, 2, 1025), (65, 511, 515), (1777, 512, 96), (3000, 10007, 40),
                                                (5000, 262143, 8), (4097, 262144, 16), (131073, 300, 9), (200000, 100000, 4)])
def test_embed_grad(dtype, tokens, vocab, width):
    dy, ids = normal((tokens, width), dtype, width), ids_of(tokens, vocab, tokens + vocab)
    got = tng.embed_grad(dy, ids, vocab, scale=0.37)
    embed_grad_check(dy, ids, vocab, 0.37, got)
    assert torch.equal(tng.embed_grad(dy, ids.to(torch.int32), vocab, scale=0.37), got)          # and the same bits each time


@pytest.mark.parametrize("tokens", [1, 31, 32, 33, 64, 1000, 20000])
@pytest.mark.parametrize("kind", ["one id", "two ids", "all empty", "sorted", "reversed", "each once", "outside"])
def test_embed_grad_of_extreme_batches(tokens, kind):
    vocab = 30000
    t = torch.arange(tokens, device="cuda")
    ids = {"one id": t * 0 + 17, "two ids": (t % 2) * (vocab - 1), "all empty": t * 0 - 1, "sorted": t // 3, "reversed": (tokens - 1 - t) // 40,
           "each once": t * 7919 % vocab, "outside": torch.where(t % 3 == 0, t, vocab + t)}[kind]
    dy = normal((tokens, 130), torch.float32, tokens)
    embed_grad_check(dy, ids, vocab, 1.0, tng.embed_grad(dy, ids, vocab))


@pytest.mark.parametrize("lead,pad", [(0, 8), (4, 4), (1, 0), (3, 5)])
def test_embed_grad_into_a_part_of_a_row(lead, pad):
    vocab, width, tokens = 201, 516, 700
    d, buf = inside(vocab, width, torch.float32, lead, width + pad)
    dy, _ = inside(tokens, width, torch.bfloat16, lead, width + pad)
    dy.copy_(normal((tokens, width), torch.bfloat16, 3))
    ids = ids_of(tokens, vocab, 4)
    tng.embed_grad(dy, ids, vocab, dtable=d)
    embed_grad_check(dy, ids, vocab, 1.0, d)
    assert untouched(buf, d)


def test_embed_grad_is_that_of_embed_by_differences():
    """Linear: y(T + e E) - y(T) pairs with dy as the gradient pairs with E, whatever e."""
    table, e = normal((50, 64), torch.float32, 1), normal((50, 64), torch.float32, 2)
    ids, dy = ids_of(200, 50, 3), normal((200, 64), torch.float32, 4)
    left = ((tng.embed(table + e, ids, scale=2.0).double() - tng.embed(table, ids, scale=2.0).double()) * dy.double()).sum()
    right = (tng.embed_grad(dy, ids, 50, scale=2.0).double() * e.double()).sum()
    # per element of y: table + e and two products round (3 u of magnitudes below 2 * 8); 12800 elements with |dy| about 0.8
    assert abs(left - right).item() < 12800 * 0.8 * 3 * U * 16 + 1e-9


# ---- norm --------------------------------------------------------------------------------------------

def norm_wanted(x, w, eps, residual):
    """h as stored, r and y in 64 bits; codes and their scale before r by fp32 steps."""
    h = x if residual is None else (x.float() + residual.float()).to(x.dtype)
    h64 = h.double()
    r = 1.0 / (h64.square().mean(1) + eps).sqrt()
    t = h.float() * w
    q, s = tng.quant8_rows(t)                               # (tested on its own)
    return h, r, h64 * r[:, None] * w.double(), q, s


def norm_check(x, w, eps, residual, y, q, scale, h, r):
    k = x.shape[1]
    want_h, want_r, want_y, want_q, want_s = norm_wanted(x, w, eps, residual)
    assert torch.equal(h, want_h)
    rel = 1.01 * (k / 2 + 4) * U                            # the mean's sum, division, sum with eps: halved by the root; its rounding
    close(r, want_r, rel * want_r)
    if y is not None:                                       # two products and the type's rounding (a step of its smallest number below that)
        close(y, want_y, ((rel + 2.02 * U) * (1 + half(y.dtype)) + half(y.dtype)) * want_y.abs() + torch.finfo(y.dtype).smallest_normal * half(y.dtype))
    if q is not None:
        assert torch.equal(q, want_q)
        close(scale, want_s.double() * want_r, (rel + 1.01 * U) * want_s.double() * want_r)


SHAPES = [(1, 1), (1, 4096), (3, 7), (9, 64), (17, 255), (5, 256), (33, 257), (700, 130), (3, 1000), (40, 1001), (2, 4097), (200, 4096), (5, 8192), (3, 9001), (2, 16384),
          (3, 16385), (2, 40000), (2000, 40)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_norm(dtype, rows, cols):
    x, residual, w = normal((rows, cols), dtype, cols), normal((rows, cols), dtype, cols + 1, 3.0), 1 + normal((cols,), torch.float32, 5, 0.1)
    for res in (None, residual):
        y, h, r = tng.rmsnorm(x, w, residual=res)
        norm_check(x, w, 1e-6, res, y, None, None, h, r)
        y8 = torch.empty_like(x)
        q, s, h8, r8 = tng.rmsnorm8(x, w, residual=res, y=y8)
        norm_check(x, w, 1e-6, res, None, q, s, h8, r8)
        assert torch.equal(y8, y) and torch.equal(r8, r)
        base = q._base if q._base is not None else q
        assert not base[:, cols:].any()                     # padding is written


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols", [(200000, 128), (40000, 1000), (8192, 4096), (4000, 8192), (2000, 16384)])
def test_many_codes(dtype, rows, cols):
    """A product and a sum rounded once instead of twice would change about one code in two million."""
    x, res, w = normal((rows, cols), dtype, 1), normal((rows, cols), dtype, 2), 1 + normal((cols,), torch.float32, 5, 0.1)
    q, s, h, r = tng.rmsnorm8(x, w, residual=res)
    want, scale = tng.quant8_rows(h.float() * w)
    assert torch.equal(q, want)
    assert torch.equal(s, scale * r)                        # (an fp32 product)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("cols", [100, 1000, 5000, 20000])
@pytest.mark.parametrize("lead,pad", [(0, 8), (8, 16), (1, 0), (3, 5), (0, 1)])
def test_norm_rows_that_start_anywhere(dtype, cols, lead, pad):
    rows, w = 21, 1 + normal((cols,), torch.float32, 5, 0.1)
    x, _ = inside(rows, cols, dtype, lead, cols + pad)
    x.copy_(normal((rows, cols), dtype, 1))
    res = normal((rows, cols), dtype, 2)
    (h, bh), (y, by) = inside(rows, cols, dtype, lead, cols + pad), inside(rows, cols, dtype, lead, cols + pad)
    q, s, _, r = tng.rmsnorm8(x, w, 1e-5, res, h=h, y=y)
    norm_check(x, w, 1e-5, res, y, q, s, h, r)
    assert untouched(bh, h) and untouched(by, y)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("cols", [64, 999, 4100, 17000])
def test_norm_in_place(dtype, cols):
    x, res, w = normal((50, cols), dtype, 1), normal((50, cols), dtype, 2), 1 + normal((cols,), torch.float32, 5, 0.1)
    want = tng.rmsnorm(x, w, residual=res)
    want8 = tng.rmsnorm8(x, w, residual=res)
    for into in ("residual", "x"):
        a, b = x.clone(), res.clone()
        got = tng.rmsnorm8(a, w, residual=b, h=b if into == "residual" else a)
        assert all(torch.equal(g, v) for g, v in zip(got, want8))
        a, b = x.clone(), res.clone()
        got = tng.rmsnorm(a, w, residual=b, h=b, y=a)
        assert all(torch.equal(g, v) for g, v in zip(got, want))
    a = x.clone()
    assert torch.equal(tng.rmsnorm(a, w, y=a)[0], tng.rmsnorm(x, w)[0])


@pytest.mark.parametrize("cols", [100, 3000, 6000, 20000])
def test_norm_rows_of_zeros_and_rows_that_are_not_finite(cols):
    x, w = normal((8, cols), torch.float32, 1), 1 + normal((cols,), torch.float32, 5, 0.1)
    x[1] = 0
    x[2, 5] = float("inf")
    x[3, 6] = float("nan")
    x[4] *= 1e25                                            # squares beyond fp32
    x[5] *= 1e-30
    q, s, h, r = tng.rmsnorm8(x, w)
    y = tng.rmsnorm(x, w)[0]
    assert not q[1].any() and s[1] == 0 and not y[1].any()
    assert not q[2].any() and not q[3].any() and not bool(s[2:4].isfinite().any()) and bool(y[3].isnan().all())
    assert r[2] == 0 and bool(y[2, 5].isnan()) and r[4] == 0 and s[4] == 0 and not y[4].any()
    rest = torch.tensor([0, 5, 6, 7], device="cuda")
    norm_check(x[rest], w, 1e-6, None, y[rest], q[rest], s[rest], h[rest], r[rest])
    half_prec = torch.full((1, cols), 60000.0, dtype=torch.float16, device="cuda")      # the sum with the residual overflows the type
    q, s, h, r = tng.rmsnorm8(half_prec, w, residual=half_prec)
    assert bool(h.isinf().all()) and not bool(s.isfinite().any())


def grad_check(dy, h, w, r, dres, dx, dw):
    k, n = dy.shape[1], dy.shape[0]
    d, h64, r64, w64 = dy.double(), h.double(), r.double()[:, None], w.double()
    g = d * w64
    dot, size = (g * h64).sum(1, keepdim=True), (g * h64).abs().sum(1, keepdim=True)
    along = h64 * r64 ** 2 / k
    want = r64 * (g - along * dot)
    res = 0 if dres is None else dres.double()
    if dx is not None:
        # the sum of k products of a product each, r r dot / k: four roundings; g, the fused product, the product with r: three
        err = r64 * (along.abs() * size * (k + 7) * 1.01 * U + g.abs() * 3.03 * U + (along * dot).abs() * 3.03 * U)
        if dres is not None:
            err = err + U * 1.01 * (want + res).abs()
        close(dx, want + res, err + half(dx.dtype) * ((want + res).abs() + err) + torch.finfo(dx.dtype).smallest_normal * half(dx.dtype))
    if dw is not None:
        terms = d * h64 * r64
        close(dw, terms.sum(0), 1.01 * (n + 2) * U * terms.abs().sum(0))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_norm_grad(dtype, rows, cols):
    h, w = normal((rows, cols), dtype, 1, 2.0), 1 + normal((cols,), torch.float32, 5, 0.1)
    dy, res = normal((rows, cols), dtype, 2, 0.1), normal((rows, cols), dtype, 3, 0.1)
    _, _, r = tng.rmsnorm(h, w)
    for dres in (None, res):
        dx, dw = tng.rmsnorm_grad(dy, h, w, r, dres=dres)
        grad_check(dy, h, w, r, dres, dx, dw)
        again = tng.rmsnorm_grad(dy, h, w, r, dres=dres)
        assert torch.equal(dx, again[0]) and torch.equal(dw, again[1])
        for into in ("dy", "dres"):
            a, b = dy.clone(), None if dres is None else dres.clone()
            if into == "dres" and b is None:
                continue
            assert torch.equal(tng.rmsnorm_grad(a, h, w, r, dres=b, dx=a if into == "dy" else b)[0], dx)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("cols", [100, 1000, 5000, 20000])
@pytest.mark.parametrize("lead,pad", [(0, 8), (1, 0), (3, 5)])
def test_norm_grad_rows_that_start_anywhere(dtype, cols, lead, pad):
    rows, w = 150, 1 + normal((cols,), torch.float32, 5, 0.1)
    views = [inside(rows, cols, dtype, lead, cols + pad) for _ in range(4)]
    dy, h, res, dx = (v for v, _ in views)
    for i, v in enumerate((dy, h, res)):
        v.copy_(normal((rows, cols), dtype, i))
    r = tng.rmsnorm(h, w)[2]
    big = torch.full((cols + 6,), 7.0, device="cuda")
    dw = big[3:3 + cols]
    tng.rmsnorm_grad(dy, h, w, r, dres=res, dx=dx, dw=dw)
    grad_check(dy, h, w, r, res, dx, dw)
    assert untouched(views[3][1], dx) and bool((big[:3] == 7).all()) and bool((big[3 + cols:] == 7).all())


@pytest.mark.parametrize("rows,cols", [(3, 100), (500, 64), (500, 1001), (500, 3000), (500, 16384), (40, 20000)])
def test_outputs_that_are_left_out(rows, cols):
    """The C calls' optional outputs, one by one."""
    x, res, w = normal((rows, cols), torch.bfloat16, 1), normal((rows, cols), torch.bfloat16, 2), 1 + normal((cols,), torch.float32, 5, 0.1)
    y = torch.empty_like(x)
    q, s, h, r = tng.rmsnorm8(x, w, residual=res, y=y)
    dx, dw = tng.rmsnorm_grad(x, h, w, r)
    st = torch.cuda.current_stream().cuda_stream
    L, P = tng.lib(), lambda t: t.data_ptr()
    ldq = -(-cols // 16) * 16
    for want in ("h", "y", "r", "q"):
        out = {"h": torch.zeros_like(h), "y": torch.zeros_like(y), "r": torch.zeros_like(r), "q": tng.empty_codes(rows, cols)}[want]
        scale = torch.zeros_like(s)
        give = lambda n: P(out) if n == want else None
        assert L.tng_rmsnorm(P(x), tng.BF16, rows, cols, cols, P(res), cols, P(w), 1e-6, give("h"), cols, give("y"), cols, give("q"), ldq,
                             P(scale) if want == "q" else None, give("r"), st) == tng.OK
        assert torch.equal(out, {"h": h, "y": y, "r": r, "q": q}[want]) and (want != "q" or torch.equal(scale, s))
    scratch = torch.empty(L.tng_rmsnorm_grad_scratch_bytes(rows, cols), dtype=torch.uint8, device="cuda")
    gx, gw = torch.zeros_like(dx), torch.zeros_like(dw)
    assert L.tng_rmsnorm_grad(P(x), cols, P(h), cols, tng.BF16, rows, cols, P(w), P(r), None, 0, P(gx), cols, None, None, st) == tng.OK
    assert L.tng_rmsnorm_grad(P(x), cols, P(h), cols, tng.BF16, rows, cols, P(w), P(r), None, 0, None, 0, P(gw), P(scratch), st) == tng.OK
    assert torch.equal(gx, dx) and torch.equal(gw, dw)


def test_norm_grad_by_differences():
    """The directional derivative of sum(y dy) in 64 bits, central differences with a step of 2^-12: off by step^2 times a third
    derivative (of the order of the gradient over h^2) and the rounding of the fp32 gradient."""
    k, w = 96, 1 + normal((96,), torch.float32, 5, 0.1)
    h, dy, e, ew = (normal((30, k), torch.float32, i) for i in (1, 2, 3, 4))
    ew = ew[0]
    r = tng.rmsnorm(h, w)[2]
    dx, dw = tng.rmsnorm_grad(dy, h, w, r)

    def f(hh, ww):
        hh, ww = hh.double(), ww.double()
        return (hh / (hh.square().mean(1, keepdim=True) + 1e-6).sqrt() * ww * dy.double()).sum().item()

    step = 2.0 ** -12
    slope = (f(h.double() + step * e.double(), w.double() + step * ew.double()) - f(h.double() - step * e.double(), w.double() - step * ew.double())) / (2 * step)
    got = (dx.double() * e.double()).sum().item() + (dw.double() * ew.double()).sum().item()
    size = (dx.double() * e.double()).abs().sum().item() + (dw.double() * ew.double()).abs().sum().item()
    assert abs(got - slope) < (200 * U + 10 * step ** 2) * size


def test_norm_of_nothing():
    w = torch.ones(20, device="cuda")
    none = torch.empty((0, 20), device="cuda")
    q, s, h, r = tng.rmsnorm8(none, w)
    assert q.shape == (0, 20) and s.shape == r.shape == (0,)
    dw = torch.full((20,), 3.0, device="cuda")
    dx, _ = tng.rmsnorm_grad(none, none, w, r, dw=dw)
    assert dx.shape == (0, 20) and not dw.any()


# ---- together ----------------------------------------------------------------------------------------

def test_norm_codes_feed_products_as_quantised_rows_would():
    """product8 of the norm's codes = the layer on the exact normed rows, up to the codes' rounding: half a step of the row's scale
    against weights that are codes too."""
    x, res, w = normal((70, 512), torch.bfloat16, 1), normal((70, 512), torch.bfloat16, 2), 1 + normal((512,), torch.float32, 5, 0.1)
    wq, ws = tng.quant8_rows(normal((300, 512), torch.float32, 3, 512 ** -0.5))
    q, s, h, r = tng.rmsnorm8(x, w, residual=res)
    got = tng.product8(q, s, wq, ws, dtype=torch.float32)
    weight = wq.double() * ws.double()[:, None]
    want = (h.double() * r.double()[:, None] * w.double()) @ weight.t()
    # |y - q s| <= s / 2 (1 + 2^-16) an element (127 steps of fp32 rounding); the product's two fp32 products
    close(got, want, s.double()[:, None] / 2 * 1.0001 * weight.abs().sum(1)[None, :] + 2.02 * U * want.abs() + 1e-12)


@pytest.mark.parametrize("other_stream", [False, True])
def test_a_captured_chain_replays_on_new_inputs(other_stream):
    vocab, width, tokens = 300, 256, 200
    table, w = normal((vocab, width), torch.float32, 1), 1 + normal((width,), torch.float32, 2, 0.1)
    ids, dy = ids_of(tokens, vocab, 3), normal((tokens, width), torch.bfloat16, 4)

    def chain(ids, dy):
        h = tng.embed(table, ids, scale=4.0, dtype=torch.bfloat16)
        q, s, h, r = tng.rmsnorm8(h, w)
        dx, dw = tng.rmsnorm_grad(dy, h, w, r)
        return q, s, dx, dw, tng.embed_grad(dx, ids, vocab, scale=4.0)

    stream = torch.cuda.Stream() if other_stream else None
    static_ids, static_dy = ids.clone(), dy.clone()
    chain(static_ids, static_dy)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        out = chain(static_ids, static_dy)
    for seed in (7, 8):
        static_ids.copy_(ids_of(tokens, vocab, seed))
        static_dy.copy_(normal((tokens, width), torch.bfloat16, seed))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, chain(static_ids, static_dy)))


def test_calls_on_two_streams_at_once():
    vocab, width, tokens = 5000, 512, 3000
    jobs = []
    for i in range(2):
        jobs.append((torch.cuda.Stream(), normal((tokens, width), torch.bfloat16, i), ids_of(tokens, vocab, i)))
    want = [tng.embed_grad(dy, ids, vocab) for _, dy, ids in jobs]
    torch.cuda.synchronize()
    for _ in range(5):
        got = []
        for stream, dy, ids in jobs:
            with torch.cuda.stream(stream):
                got.append(tng.embed_grad(dy, ids, vocab))
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_embed_grad_of_a_long_batch():
    """Chunks longer than what a block looks up at a time."""
    tokens, vocab = 1300000, 50
    dy, ids = normal((tokens, 5), torch.float32, 1), ids_of(tokens, vocab, 2, torch.int32)
    embed_grad_check(dy, ids, vocab, 1.0, tng.embed_grad(dy, ids, vocab))


def test_gradients_of_empty_places_may_be_anything():
    dy, ids = normal((500, 96), torch.bfloat16, 1), ids_of(500, 40, 2)
    ids[::7] = -1
    want = tng.embed_grad(dy, ids, 40)
    dy[ids < 0] = float("nan")
    assert torch.equal(tng.embed_grad(dy, ids, 40), want)
    want = tng.embed(dy, torch.full((3,), -1, device="cuda"))
    assert not want.any()                                   # zeros, whatever the table holds


def test_offsets_beyond_32_bits():
    ld = (1 << 31) + 64                                     # elements of bf16: rows 4 GB apart
    buf = torch.zeros(ld + 4096, dtype=torch.bfloat16, device="cuda")
    far = buf.as_strided((2, 4096), (ld, 1))
    far.copy_(normal((2, 4096), torch.bfloat16, 1))
    near, w = far.contiguous(), 1 + normal((4096,), torch.float32, 2, 0.1)
    ids = torch.tensor([1, 0, 1], device="cuda")
    assert torch.equal(tng.embed(far, ids), near[ids])
    assert all(torch.equal(a, b) for a, b in zip(tng.rmsnorm8(far, w), tng.rmsnorm8(near, w)))
    r = tng.rmsnorm(near, w)[2]
    assert all(torch.equal(a, b) for a, b in zip(tng.rmsnorm_grad(far, near, w, r), tng.rmsnorm_grad(near, near, w, r)))
    assert torch.equal(tng.embed_grad(far, ids[:2], 3), tng.embed_grad(near, ids[:2], 3))
    out = torch.empty_like(near)
    tng.rmsnorm(near, w, y=far)
    tng.rmsnorm(near, w, y=out)
    assert torch.equal(far, out)
    del buf, far
    ld = (1 << 30) + 64                                     # of fp32
    buf = torch.full((ld + 64,), 5.0, device="cuda")
    d = buf.as_strided((2, 33), (ld, 1))
    tng.embed_grad(near[:, :33], ids[:2], 2, dtable=d)
    assert torch.equal(d, near[:, :33].float().flip(0)) and bool((buf[33:64] == 5).all()) and bool((buf[ld + 33:] == 5).all())


def test_refusals():
    x, w = normal((4, 32), torch.bfloat16, 1), torch.ones(32, device="cuda")
    ids = torch.zeros(4, dtype=torch.int64, device="cuda")
    with pytest.raises(TypeError):
        tng.rmsnorm(x, w.bfloat16())
    with pytest.raises(TypeError):
        tng.rmsnorm(x, w[:31])
    with pytest.raises(TypeError):
        tng.rmsnorm(x, w, residual=x.float())
    with pytest.raises(ValueError):
        tng.rmsnorm(x, w, residual=x[:3])
    with pytest.raises(ValueError):
        tng.rmsnorm(x.t(), w)
    with pytest.raises(ValueError):
        tng.rmsnorm8(x, w, q=torch.empty((4, 40), dtype=torch.int8, device="cuda")[:, 1:33].contiguous()[:, :31])
    for eps in (0.0, -1.0, float("nan"), float("inf")):
        with pytest.raises(tng.TngError):
            tng.rmsnorm(x, w, eps=eps)
    with pytest.raises(TypeError):
        tng.embed(x, ids.float())
    with pytest.raises(ValueError):
        tng.embed(x, ids.view(2, 2))
    with pytest.raises(ValueError):
        tng.embed(x, torch.zeros(8, dtype=torch.int64, device="cuda")[::2])
    with pytest.raises(TypeError):
        tng.embed(x, ids.cpu())
    with pytest.raises(TypeError):
        tng.embed(x, ids, dtype=torch.float32, out=torch.empty_like(x))
    with pytest.raises(ValueError):
        tng.embed_grad(x, ids[:3], 10)
    with pytest.raises(ValueError):
        tng.embed_grad(x, ids, 10, dtable=torch.empty((10, 31), device="cuda"))
    with pytest.raises(ValueError):
        tng.embed_grad(x, ids, 10, scratch=torch.empty(16, dtype=torch.uint8, device="cuda"))
