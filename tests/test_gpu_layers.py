"""8-bit linear layers and dropout on the GPU against the plain restatement.  Codes, scales, products and dropout
are unique (every decision is a stated sequence of fp32 operations, the integer sums are exact), so they are
compared bit for bit; db is an fp32 sum, compared with the 64-bit one."""
import numpy as np
import pytest
import torch

import layers_ref as ref
from gpu_util import to_np
from paper_1901_08227_b200 import tng

pytestmark = pytest.mark.gpu

DTYPES = [torch.float32, torch.bfloat16, torch.float16]
SEED = 0x0123456789ABCDEF


def values(shape, dtype, seed, scale=1.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


def strided(x, pad):
    """The same values with a row stride of cols + pad, starting `pad % 4` elements into the buffer."""
    rows, cols = x.shape
    buf = torch.full((rows * (cols + pad) + 8,), float("nan"), dtype=x.dtype, device=x.device)
    v = buf[pad % 4:pad % 4 + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    v.copy_(x)
    return v


def f32(t):
    return t.float().cpu().numpy()


def rounded(y, dtype):
    """A float32 array rounded once to dtype, back in float32."""
    return torch.from_numpy(np.ascontiguousarray(y)).to(dtype).float().numpy()


def same(a, b):
    return np.array_equal(a, b, equal_nan=True)


def uni(rows, cols, d, tag):
    return ref.uniforms(rows, cols, d.seed_lo | d.seed_hi << 32, d.layer, d.step, tag, d.row0)


# ---- quantiser -----------------------------------------------------------------------------------
SHAPES = [(1, 1), (1, 7), (3, 8), (5, 129), (33, 1000), (130, 1024), (7, 1025), (17, 4096), (2, 16384), (1, 20001), (513, 65)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("pad", [None, 0, 3, 8])
def test_codes_by_row_and_by_column(dtype, rows, cols, pad):
    x = values((rows, cols), dtype, rows * 1000 + cols)
    if rows > 2:
        x[1] = 0
    if cols > 2:
        x[:, 2] = 0
    if pad is not None:
        x = strided(x, pad)
    xn = f32(x)
    for draw in (None, tng.Draw(SEED, 5, 77, row0=3)):
        u = None if draw is None else uni(rows, cols, draw, ref.TAG_ROUNDING)
        q, s = tng.quant8_rows(x, draw)
        wq, ws = ref.codes(xn, u)
        assert same(to_np(q), wq) and same(to_np(s), ws)
        colsum = torch.empty(cols, device="cuda")
        q, s = tng.quant8_cols(x, draw, colsum=colsum)
        wq, ws = ref.codes(xn.T, None if u is None else u.T)
        assert same(to_np(q), wq) and same(to_np(s), ws)
        x64 = xn.astype(np.float64)
        # a sum of n fp32 numbers in any order: off by at most n 2^-24 of the sum of magnitudes
        assert np.all(np.abs(to_np(colsum) - x64.sum(0)) <= rows * 2.0 ** -24 * np.abs(x64).sum(0))


def test_padding_of_codes_is_zero():
    x = values((70, 45), torch.bfloat16, 1)
    for rows, cols, make in [(70, 45, tng.quant8_rows), (45, 70, tng.quant8_cols)]:
        buf = torch.full((rows, -(-cols // 16) * 16), 99, dtype=torch.int8, device="cuda")
        make(x, q=buf[:, :cols])
        assert not to_np(buf)[:, cols:].any()


@pytest.mark.parametrize("dtype", DTYPES)
def test_lines_that_are_zero_tiny_or_not_finite(dtype):
    x = values((12, 300), dtype, 3)
    x[0] = 0
    x[1, 5] = float("nan")
    x[2, 6] = float("inf")
    x[3, 299] = float("-inf")
    x[4] = torch.finfo(dtype).max
    x[5] = -torch.finfo(dtype).max
    x[6] = 0
    x[6, 1] = torch.finfo(dtype).smallest_normal
    if dtype != torch.float16:
        x[7] *= 2.0 ** -118
        x[8] *= 2.0 ** -126
    for draw in (None, tng.Draw(1, 2, 3)):
        u = None if draw is None else uni(12, 300, draw, ref.TAG_ROUNDING)
        q, s = tng.quant8_rows(x, draw)
        wq, ws = ref.codes(f32(x), u)
        assert same(to_np(q), wq) and same(to_np(s), ws)
        q, s = tng.quant8_cols(x.t().contiguous(), draw)
        u = None if draw is None else uni(300, 12, draw, ref.TAG_ROUNDING).T
        wq, ws = ref.codes(f32(x), u)
        assert same(to_np(q), wq) and same(to_np(s), ws)
    # a product never hides a value that is not finite
    w, sw = tng.quant8_rows(values((4, 300), dtype, 4))
    y = f32(tng.linear8(x, w, sw))
    assert np.all(np.isnan(y[1:4])) and not np.any(np.isnan(y[[0, 6]])) and not y[0].any()


def test_a_part_of_a_batch_draws_what_the_whole_batch_does():
    x = values((40, 100), torch.float32, 9)
    whole, _ = tng.quant8_rows(x, tng.Draw(SEED, 1, 2))
    part, _ = tng.quant8_rows(x[25:], tng.Draw(SEED, 1, 2, row0=25))
    assert torch.equal(whole[25:], part)
    whole = tng.dropout(x, 0.4, tng.Draw(SEED, 1, 2))
    assert torch.equal(whole[25:], tng.dropout(x[25:], 0.4, tng.Draw(SEED, 1, 2, row0=25)))
    last = tng.Draw(SEED, 1, 2, row0=(1 << 32) - 40)
    u = uni(40, 100, last, ref.TAG_DROPOUT)
    assert same(f32(tng.dropout(x, 0.4, last)), ref.dropout(f32(x), 0.4, u))


# ---- product ---------------------------------------------------------------------------------------
def random_codes(lines, n, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    q = tng.empty_codes(lines, n)
    q.copy_(torch.randint(-127, 128, (lines, n), generator=g, device="cuda"))
    s = torch.rand(lines, generator=g, device="cuda") * 0.01 + 1e-4
    return q, s


PRODUCTS = [(1, 1, 1), (1, 128, 16), (1, 4096, 4096), (2, 100, 333), (3, 1001, 4097), (7, 515, 129), (8, 4096, 2048), (9, 200, 1000), (16, 256, 256),
            (17, 300, 4096), (31, 64, 65), (64, 1024, 1024), (65, 127, 15), (127, 129, 128), (128, 128, 128), (129, 257, 513), (200, 2503, 1001),
            (256, 256, 4096), (257, 512, 127), (300, 1, 40), (511, 513, 777), (640, 4096, 100), (1000, 1000, 1000), (1333, 2503, 1001), (2048, 2048, 512),
            (2500, 1700, 16), (5, 70, 131056), (130, 140, 131056), (300, 260, 20000)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,n,k", PRODUCTS)
def test_product(dtype, m, n, k):
    a, sa = random_codes(m, k, m + 7 * k)
    b, sb = random_codes(n, k, n + 11 * k)
    bias = values((n,), torch.float32, 5) if (m + n) % 2 else None
    out = tng.product8(a, sa, b, sb, bias=bias, dtype=dtype)
    acc = (a.double() @ b.double().t()).round()                     # exact: below 2^53
    y = acc.float() * sa[:, None] * sb[None, :]                     # one fp32 rounding each
    if bias is not None:
        y = y + bias
    assert torch.equal(out, y.to(dtype))


@pytest.mark.parametrize("m", [1, 5, 40, 300])
def test_product_of_extreme_codes_is_exact(m):
    # the largest sum the contraction limit allows: 128 * 128 * 131056 < 2^31
    k, n = 131056, 130
    a = torch.full((m, k), -128, dtype=torch.int8, device="cuda")
    b = torch.full((n, k), -128, dtype=torch.int8, device="cuda")
    one = torch.ones(max(m, n), device="cuda")
    out = tng.product8(a, one[:m], b, one[:n], dtype=torch.float32)
    assert torch.equal(out, torch.full((m, n), 128.0 * 128 * k, device="cuda"))
    b[1::2] = 127
    out = tng.product8(a, one[:m], b, one[:n], dtype=torch.float32)
    assert torch.equal(out[:, 1], torch.full((m,), -128.0 * 127 * k, device="cuda"))


@pytest.mark.parametrize("m", [1, 6, 33, 260])
@pytest.mark.parametrize("dtype,pad", [(torch.float32, 1), (torch.float32, 4), (torch.bfloat16, 3), (torch.bfloat16, 8), (torch.float16, 5)])
def test_product_into_strided_rows_writes_nothing_else(m, dtype, pad):
    n, k = 301, 200
    a, sa = random_codes(m, k + 32, 1)
    b, sb = random_codes(n, k + 16, 2)
    a, b = a[:, :k], b[:, :k]                                       # what follows a line must not count
    out = strided(torch.zeros((m, n), dtype=dtype, device="cuda"), pad)
    base = out.as_strided((m, n + pad), (n + pad, 1))
    base[:, n:] = 7
    tng.product8(a, sa, b, sb, out=out)
    want = tng.product8(a, sa, b, sb, dtype=dtype)
    y = (a.double() @ b.double().t()).float() * sa[:, None] * sb[None, :]
    assert torch.equal(out, want) and torch.equal(want, y.to(dtype)) and bool((base[:, n:] == 7).all())


# ---- linear layer ----------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T,K,N", [(1, 64, 48), (1, 4096, 1000), (1, 4099, 130), (2, 20001, 65), (4, 300, 129), (8, 2048, 512), (9, 77, 200), (33, 1001, 515),
                                   (150, 513, 300), (515, 1024, 256)])
def test_linear_forward(dtype, T, K, N):
    x = values((T, K), dtype, T + K)
    if T > 3:
        x[2] = 0
    w, sw = tng.quant8_rows(values((N, K), torch.float32, 6, K ** -0.5))
    bias = values((N,), torch.float32, 8)
    for b in (None, bias):
        want = rounded(ref.linear(f32(x), to_np(w), to_np(sw), None if b is None else to_np(b)), dtype)
        assert same(f32(tng.linear8(x, w, sw, bias=b)), want)
        assert same(f32(tng.linear8(strided(x, 3), w, sw, bias=b)), want)
    # what the caller's scratch held before makes no difference
    scratch = torch.full((tng.lib().tng_linear8_scratch_bytes(T, K) + 256,), 0xA5, dtype=torch.uint8, device="cuda")
    assert same(f32(tng.linear8(x, w, sw, bias=bias, scratch=scratch)), want)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T,K,N", [(1, 20, 30), (2, 130, 65), (17, 128, 128), (64, 257, 1000), (129, 1000, 515), (777, 333, 260), (1030, 512, 640)])
@pytest.mark.parametrize("drawn", [False, True])
def test_linear_gradients(dtype, T, K, N, drawn):
    x, dy = values((T, K), dtype, 1), values((T, N), dtype, 2, 1e-2)
    if T > 5:
        dy[3:5] = 0                                                 # masked tokens
    w = values((N, K), torch.float32, 3, K ** -0.5)
    wt, swt = tng.quant8_cols(w)
    d = tng.Draw(SEED, 9, 4, row0=6) if drawn else None
    u = uni(T, N, d, ref.TAG_ROUNDING) if drawn else None
    scratch = torch.full((tng.lib().tng_linear8_grad_scratch_bytes(T, K, N),), 0xA5, dtype=torch.uint8, device="cuda")
    dx, dw, db = tng.linear8_grad(dy, x, wt, swt, draw=d, scratch=scratch)
    wdx, wdw, wdb = ref.linear_grad(f32(dy), f32(x), to_np(wt), to_np(swt), u)
    assert same(f32(dx), rounded(wdx, dtype))
    assert same(to_np(dw), wdw)
    mag = np.abs(f32(dy).astype(np.float64)).sum(0)
    assert np.all(np.abs(to_np(db) - wdb) <= T * 2.0 ** -24 * mag)
    # into a worker's row of gradients, inputs strided
    row = torch.full((N * (K + 5) + 16,), float("nan"), device="cuda")
    view = row[4:4 + N * (K + 5)].view(N, K + 5)[:, :K]
    dx2, _, db2 = tng.linear8_grad(strided(dy, 3), strided(x, 1), wt, swt, draw=d, dw=view, dx=strided(torch.zeros_like(x), 5))
    assert torch.equal(view, dw) and torch.equal(dx2, dx) and np.isnan(to_np(row[4:4 + N * (K + 5)].view(N, K + 5)[:, K:])).all()
    assert np.all(np.abs(to_np(db2) - wdb) <= T * 2.0 ** -24 * mag)


def test_linear_gradients_match_differences():
    """sum(dy * y) is linear in x and W; its difference quotients (64 bits) against dx and dw, within what coding may change."""
    T, K, N = 40, 96, 72
    x, w, dy = (to_np(values(s, torch.float32, i)).astype(np.float64) for i, s in enumerate([(T, K), (N, K), (T, N)]))
    wt, swt = tng.quant8_cols(torch.from_numpy(w).float().cuda())
    dx, dw, db = tng.linear8_grad(torch.from_numpy(dy).float().cuda(), torch.from_numpy(x).float().cuda(), wt, swt)
    rng = np.random.default_rng(0)
    h = 0.25
    for which, base, got in (("x", x, to_np(dx)), ("w", w, to_np(dw))):
        for _ in range(20):
            at = tuple(rng.integers(0, n) for n in base.shape)
            e = np.zeros_like(base)
            e[at] = h
            f = (lambda v: (dy * (v @ w.T)).sum()) if which == "x" else (lambda v: (dy * (x @ v.T)).sum())
            fd = (f(base + e) - f(base - e)) / (2 * h)
            p, q = (dy[at[0]], w[:, at[1]]) if which == "x" else (dy[:, at[0]], x[:, at[1]])
            sp = np.abs(p).max() / 127
            sq = np.abs(q).max() / 127
            assert abs(got[at] - fd) <= 1.01 * (np.abs(p) * sq / 2 + np.abs(q) * sp / 2 + sp * sq / 4).sum()


def test_parts_of_the_gradient_can_be_left_out():
    T, K, N = 33, 64, 80
    x, dy = values((T, K), torch.bfloat16, 1), values((T, N), torch.bfloat16, 2)
    wt, swt = tng.quant8_cols(values((N, K), torch.float32, 3))
    dx, dw, db = tng.linear8_grad(dy, x, wt, swt)
    L, st = tng.lib(), torch.cuda.current_stream().cuda_stream
    buf = torch.empty(L.tng_linear8_grad_scratch_bytes(T, K, N), dtype=torch.uint8, device="cuda")
    for want in ("x", "w", "b", "wb", "xb"):
        ox, ow, ob = torch.zeros_like(dx), torch.zeros_like(dw), torch.zeros_like(db)
        has_x, has_w = "x" in want, "w" in want
        assert L.tng_linear8_grad(dy.data_ptr(), N, x.data_ptr() if has_w else None, K, tng.BF16, T, K, N, wt.data_ptr() if has_x else None,
                                  wt.stride(0), swt.data_ptr() if has_x else None, None, ox.data_ptr() if has_x else None, K,
                                  ow.data_ptr() if has_w else None, K, ob.data_ptr() if "b" in want else None, buf.data_ptr(), st) == tng.OK
        assert torch.equal(ox, dx if has_x else torch.zeros_like(dx))
        assert torch.equal(ow, dw if has_w else torch.zeros_like(dw))
        assert torch.equal(ob, db if "b" in want else torch.zeros_like(db))


def test_empty_batches():
    w, sw = tng.quant8_rows(values((30, 20), torch.float32, 1))
    wt, swt = tng.quant8_cols(values((30, 20), torch.float32, 1))
    x, dy = torch.empty((0, 20), device="cuda"), torch.empty((0, 30), device="cuda")
    assert tng.linear8(x, w, sw).shape == (0, 30)
    dw = torch.full((30, 25), 5.0, device="cuda")
    _, _, db = tng.linear8_grad(dy, x, wt, swt, dw=dw[:, :20])
    assert not dw[:, :20].any() and not db.any() and bool((dw[:, 20:] == 5).all())
    assert tng.dropout(x, 0.5, tng.Draw()).shape == (0, 20)
    q, s = tng.quant8_rows(x)
    assert q.shape == (0, 20) and s.shape == (0,)
    colsum = torch.full((20,), 5.0, device="cuda")
    q, s = tng.quant8_cols(x, colsum=colsum)
    assert q.shape == (20, 0) and not s.any() and not colsum.any()


# ---- dropout -----------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 4096), (3, 5), (16, 1024), (33, 127), (5, 128), (64, 129), (257, 1001), (2, 20003)])
@pytest.mark.parametrize("p", [0.0, 0.1, 0.5, 1.0])
def test_dropout(dtype, rows, cols, p):
    x, r = values((rows, cols), dtype, 1), values((rows, cols), dtype, 2)
    if cols > 4:
        x[0, :3] = torch.tensor([float("nan"), float("inf"), -0.0], dtype=dtype)
    d = tng.Draw(SEED, 3, 12, row0=9)
    u = uni(rows, cols, d, ref.TAG_DROPOUT)
    for res in (None, r):
        want = rounded(ref.dropout(f32(x), p, u, None if res is None else f32(res)), dtype)
        assert same(f32(tng.dropout(x, p, d, residual=res)), want)
        for pad in (3, 8):
            out = strided(torch.zeros_like(x), pad)
            tng.dropout(strided(x, pad), p, d, residual=None if res is None else strided(res, pad), out=out)
            assert same(f32(out), want)
        y = x.clone()
        tng.dropout(y, p, d, residual=res, out=y)                   # in place
        assert same(f32(y), want)
    assert same(f32(tng.dropout_grad(x, p, d)), rounded(ref.dropout(f32(x), p, u), dtype))


def test_dropout_gradient_matches_differences():
    x, dy = values((20, 50), torch.float32, 1), values((20, 50), torch.float32, 2)
    d = tng.Draw(4, 5, 6)
    g = to_np(tng.dropout_grad(dy, 0.5, d)).astype(np.float64)

    def f(v):
        return (dy.double() * tng.dropout(v, 0.5, d).double()).sum().item()

    for at in [(0, 0), (3, 11), (19, 49), (7, 8)]:
        e = torch.zeros_like(x)
        e[at] = 0.5
        # x +- e and the products by 2 are rounded to fp32: an error of at most 4 |dy| 2^-23 max|x| in the quotient
        assert abs(g[at] - (f(x + e) - f(x - e))) <= 1e-5


# ---- around the calls ----------------------------------------------------------------------------------
def test_another_stream():
    x = values((300, 500), torch.bfloat16, 1)
    w, sw = tng.quant8_rows(values((400, 500), torch.float32, 2))
    wt, swt = tng.quant8_cols(values((400, 500), torch.float32, 2))
    dy = values((300, 400), torch.bfloat16, 3)
    d = tng.Draw(1, 1, 1)
    here = [tng.linear8(x, w, sw), *tng.linear8_grad(dy, x, wt, swt, draw=d), tng.dropout(x, 0.3, d)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        there = [tng.linear8(x, w, sw), *tng.linear8_grad(dy, x, wt, swt, draw=d), tng.dropout(x, 0.3, d)]
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(here, there))


def test_calls_can_be_captured_in_a_graph():
    x = values((40, 512), torch.bfloat16, 1)
    w, sw = tng.quant8_rows(values((256, 512), torch.float32, 2))
    out, y = torch.empty((40, 256), dtype=torch.bfloat16, device="cuda"), torch.empty((40, 256), dtype=torch.bfloat16, device="cuda")
    scratch = torch.empty(tng.lib().tng_linear8_scratch_bytes(40, 512), dtype=torch.uint8, device="cuda")
    d = tng.Draw(1, 2, 3)
    tng.linear8(x, w, sw, out=out, scratch=scratch)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        tng.linear8(x, w, sw, out=out, scratch=scratch)
        tng.dropout(out, 0.2, d, out=y)
    x.copy_(values((40, 512), torch.bfloat16, 5))
    graph.replay()
    want = tng.linear8(x, w, sw)
    assert torch.equal(out, want) and torch.equal(y, tng.dropout(want, 0.2, d))


@pytest.mark.parametrize("what", ["rows", "product", "dropout"])
def test_offsets_beyond_32_bits(what):
    # two rows more than 2^32 bytes apart (2^31 elements and up)
    ld = (1 << 31) + 64
    buf = torch.empty(ld + 4096, dtype=torch.bfloat16, device="cuda")
    far = buf.as_strided((2, 500), (ld, 1))
    x = values((2, 500), torch.bfloat16, 1)
    far.copy_(x)
    if what == "rows":
        q, s = tng.quant8_rows(far)
        wq, ws = ref.codes(f32(x))
        assert same(to_np(q), wq) and same(to_np(s), ws)
        q, s = tng.quant8_cols(far)
        wq, ws = ref.codes(f32(x).T)
        assert same(to_np(q), wq) and same(to_np(s), ws)
    elif what == "product":
        a, sa = random_codes(2, 64, 1)
        b, sb = random_codes(500, 64, 2)
        tng.product8(a, sa, b, sb, out=far)
        assert torch.equal(far, tng.product8(a, sa, b, sb))
    else:
        d = tng.Draw(1, 1, 1)
        assert torch.equal(tng.dropout(far, 0.5, d), tng.dropout(x, 0.5, d))
        out = buf.as_strided((2, 500), (ld, 1))
        tng.dropout(x, 0.5, d, out=out)
        assert torch.equal(out, tng.dropout(x, 0.5, d))


def refuses(f, *errors):
    with pytest.raises(errors or (tng.TngError, TypeError, ValueError)):
        f()


def test_refusals():
    x = values((8, 64), torch.bfloat16, 1)
    w, sw = tng.quant8_rows(values((32, 64), torch.float32, 2))
    a, sa = tng.quant8_rows(x)
    d = tng.Draw()
    refuses(lambda: tng.linear8(x.double(), w, sw))
    refuses(lambda: tng.linear8(x.cpu(), w, sw))
    refuses(lambda: tng.linear8(x.t(), w, sw))
    refuses(lambda: tng.linear8(x[:, :32], w, sw))
    refuses(lambda: tng.linear8(x, w, sw[:31]))
    refuses(lambda: tng.linear8(x, w, sw.double()))
    refuses(lambda: tng.linear8(x, w, sw, bias=torch.zeros(31, device="cuda")))
    refuses(lambda: tng.linear8(x, w, sw, out=torch.empty((8, 32), device="cuda")))
    x20 = values((20, 64), torch.bfloat16, 1)
    refuses(lambda: tng.linear8(x20, w, sw, scratch=torch.empty(8, dtype=torch.uint8, device="cuda")))
    refuses(lambda: tng.linear8(x[:1].expand(8, 64), w, sw), tng.TngError)          # rows that overlap
    odd = torch.zeros((32, 65), dtype=torch.int8, device="cuda")
    refuses(lambda: tng.linear8(x, odd[:, :64], sw), tng.TngError)                  # codes off their 16-byte rows
    flat = torch.zeros(32 * 64 + 16, dtype=torch.int8, device="cuda")
    refuses(lambda: tng.linear8(x, flat[1:1 + 32 * 64].view(32, 64), sw), tng.TngError)
    wide = torch.zeros((2, 131072), dtype=torch.int8, device="cuda")
    one = torch.ones(2, device="cuda")
    refuses(lambda: tng.product8(wide, one, wide, one), tng.TngError)               # contraction too long for int32
    refuses(lambda: tng.product8(a, sa, w, sw, out=torch.empty((8, 31), dtype=torch.bfloat16, device="cuda")))
    for p in (-0.1, 1.1, float("nan")):
        refuses(lambda: tng.dropout(x, p, d), tng.TngError)
    refuses(lambda: tng.dropout(x, 0.5, None), tng.TngError)
    refuses(lambda: tng.dropout(x, 0.5, tng.Draw(row0=(1 << 32) - 7)), tng.TngError)
    refuses(lambda: tng.dropout(x, 0.5, d, residual=x.float()))
    refuses(lambda: tng.dropout(x, 0.5, d, residual=x[:7]))
    refuses(lambda: tng.quant8_rows(x, tng.Draw(row0=1 << 32)), tng.TngError)
    refuses(lambda: tng.quant8_cols(x, scratch=torch.empty(8, dtype=torch.uint8, device="cuda")))
    for bad in (dict(seed=1 << 64), dict(seed=-1), dict(layer=1 << 30), dict(step=1 << 32), dict(row0=(1 << 32) + 1)):
        refuses(lambda: tng.Draw(**bad), ValueError)
    L, st = tng.lib(), torch.cuda.current_stream().cuda_stream
    raw = tng.Draw()
    raw.layer = 1 << 30
    assert L.tng_dropout(x.data_ptr(), tng.BF16, 8, 64, 64, None, 0, 0.5, raw, x.data_ptr(), 64, st) == tng.ERR_INVALID_ARG
    assert L.tng_dropout(x.data_ptr(), 3, 8, 64, 64, None, 0, 0.5, d, x.data_ptr(), 64, st) == tng.ERR_INVALID_ARG
    assert L.tng_dropout(x.data_ptr() + 1, tng.BF16, 8, 63, 64, None, 0, 0.5, d, x.data_ptr(), 64, st) == tng.ERR_INVALID_ARG
    assert L.tng_dropout(None, tng.BF16, 8, 64, 64, None, 0, 0.5, d, x.data_ptr(), 64, st) == tng.ERR_INVALID_ARG
    assert L.tng_dropout(x.data_ptr(), tng.BF16, 8, 0, 64, None, 0, 0.5, d, x.data_ptr(), 64, st) == tng.ERR_INVALID_ARG
    assert L.tng_dropout(x.data_ptr(), tng.BF16, 8, 64, 63, None, 0, 0.5, d, x.data_ptr(), 64, st) == tng.ERR_INVALID_ARG
    assert L.tng_quant8_cols(x.data_ptr(), tng.BF16, 8, 64, 64, None, a.data_ptr(), 16, sa.data_ptr(), None, None, st) == tng.ERR_INVALID_ARG
    assert L.tng_linear8(x20.data_ptr(), tng.BF16, 20, 64, 64, w.data_ptr(), 64, sw.data_ptr(), 32, None, x.data_ptr(), 32, None, st) == tng.ERR_INVALID_ARG


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T,K,N", [(129, 129 * 4, 136), (2048, 512, 520), (640, 8192, 6000), (5000, 1024, 1032), (300, 2600, 2600), (9000, 768, 2900), (1500, 5000, 20000)])
def test_linear_gradients_of_many_tiles(dtype, T, K, N):
    """dx and dw in one launch where both are whole tiles: every order of the two, all tiles written once.  The reference
    runs on the GPU in 64 bits."""
    x, dy = values((T, K), dtype, 1), values((T, N), dtype, 2, 1e-2)
    wt, swt = tng.quant8_cols(values((N, K), torch.float32, 3, K ** -0.5))
    dx = torch.full((T, K), float("nan"), dtype=dtype, device="cuda")
    dw = torch.full((N, K), float("nan"), device="cuda")
    tng.linear8_grad(dy, x, wt, swt, dx=dx, dw=dw)
    for out, (a, sa), (b, sb) in ((dx, tng.quant8_rows(dy), (wt, swt)), (dw, tng.quant8_cols(dy), tng.quant8_cols(x))):
        y = (a.double() @ b.double().t()).round().float() * sa[:, None] * sb[None, :]
        assert torch.equal(out, y.to(out.dtype))
