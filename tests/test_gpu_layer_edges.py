"""Layer operators at the edges of their tiles, launches and buffers (see test_gpu_layers.py for the operators themselves)."""
import pytest
import torch

import layers_ref as ref
from gpu_util import to_np
from paper_1901_08227_b200 import tng
from test_gpu_layers import DTYPES, SEED, f32, random_codes, rounded, same, values

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


# Around the rule between the two kernels for up to 64 rows: rows 32, 33, 64, 65 with tiles below and above half a wave and a wave.
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m", [32, 33, 64, 65])
@pytest.mark.parametrize("n,k", [(9215, 300), (9473, 300), (4863, 1200), (4609, 1200), (18944, 144), (18945, 144), (4096, 4096)])
def test_products_around_the_choice_of_a_kernel(dtype, m, n, k):
    a, sa = random_codes(m, k, m + k)
    b, sb = random_codes(n, k, n + k)
    bias = values((n,), torch.float32, 5)
    assert torch.equal(tng.product8(a, sa, b, sb, bias=bias, dtype=dtype), (wanted(a, sa, b, sb, torch.float32) + bias).to(dtype))


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


def test_an_empty_batch_clears_rows_that_are_far_apart():
    ld = (1 << 29) + 64                                     # rows 2 GB apart
    buf = torch.full((ld + 64,), 5.0, device="cuda")
    dw = buf.as_strided((2, 20), (ld, 1))
    wt, swt = tng.quant8_cols(torch.randn(2, 20, device="cuda"))
    tng.linear8_grad(torch.empty((0, 2), device="cuda"), torch.empty((0, 20), device="cuda"), wt, swt, dw=dw)
    assert not dw.any() and bool((buf[20:64] == 5).all()) and bool((buf[ld + 20:] == 5).all())


@pytest.mark.parametrize("call", ["quant8_rows", "quant8_cols", "product8", "linear8", "dropout"])
def test_a_call_that_fails_leaves_no_error_behind(call):
    """Enqueueing on the legacy stream while a stream that it synchronises with is captured is refused by the runtime; the next
    call must not report it again."""
    rt = pytest.importorskip("cuda.bindings.runtime")
    x = torch.randn(20, 64, device="cuda")
    q, s = tng.quant8_rows(x)
    qc, sc = tng.quant8_cols(x)
    y, scratch = torch.empty(20, 20, device="cuda"), torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    w, v = torch.zeros(64, device="cuda"), torch.ones(64, device="cuda")
    make = {"quant8_rows": lambda: tng.quant8_rows(x, q=q, scale=s), "quant8_cols": lambda: tng.quant8_cols(x, q=qc, scale=sc, scratch=scratch),
            "product8": lambda: tng.product8(q, s, q, s, out=y), "linear8": lambda: tng.linear8(x, q, s, out=y, scratch=scratch),
            "dropout": lambda: tng.dropout(x, 0.5, tng.Draw(), out=x)}[call]
    make()
    torch.cuda.synchronize()
    assert torch.cuda.current_stream().cuda_stream == 0
    error, stream = rt.cudaStreamCreate()
    assert error == 0 and rt.cudaStreamBeginCapture(stream, rt.cudaStreamCaptureMode.cudaStreamCaptureModeRelaxed)[0] == 0
    try:
        with pytest.raises(tng.TngError) as e:
            make()
    finally:
        rt.cudaStreamEndCapture(stream)
        rt.cudaStreamDestroy(stream)
    assert e.value.status == tng.ERR_CUDA
    tng.sgd_update(w, v, 0.5)                               # (reports whatever error its thread has pending)
    assert bool((w == -0.5).all())


# Rows of the output start on 16-byte boundaries; where they end on one too they leave by tiled copies, else by scalar stores.
# Neither may touch the padding.  (rows, columns, contraction): split in four, in two, whole tiles, several waves of them
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,n,k", [(200, 301, 4096), (1300, 4093, 2048), (300, 301, 200), (515, 1003, 777), (2570, 5121, 130), (200, 304, 4096), (1300, 4088, 2048), (300, 264, 200), (2570, 5128, 130)])
def test_products_into_padded_aligned_rows(dtype, m, n, k):
    a, sa = random_codes(m, k, m)
    b, sb = random_codes(n, k, n)
    bias = values((n,), torch.float32, 5)
    want = (wanted(a, sa, b, sb, torch.float32) + bias).to(dtype)
    for ld in (-(-n // 8) * 8, -(-n // 8) * 8 + 24):
        base = torch.full((m + 1, ld), 7.0, dtype=dtype, device="cuda")
        tng.product8(a, sa, b, sb, bias=bias, out=base[:m, :n])
        assert torch.equal(base[:m, :n], want) and bool((base[:m, n:] == 7).all()) and bool((base[m] == 7).all())
    loose = torch.full((m, n + 1), 7.0, dtype=dtype, device="cuda")       # the same by scalar stores
    if (n + 1) * loose.element_size() % 16 != 0:
        tng.product8(a, sa, b, sb, bias=bias, out=loose[:, :n])
        assert torch.equal(loose[:, :n], want) and bool((loose[:, n] == 7).all())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("drawn", [False, True])
@pytest.mark.parametrize("T,K,N", [(2050, 517, 525), (333, 301, 205), (5000, 1029, 1037), (2050, 520, 528), (333, 304, 205),
                                   (5000, 1032, 1037)])
def test_gradients_into_padded_aligned_rows(dtype, drawn, T, K, N):
    """The reference runs on the GPU in 64 bits, from the quantisers' codes."""
    x, dy = values((T, K), dtype, 1), values((T, N), dtype, 2, 1e-2)
    wt, swt = tng.quant8_cols(values((N, K), torch.float32, 3, K ** -0.5))
    d = tng.Draw(SEED, 4, 8, row0=5) if drawn else None
    ld = -(-K // 8) * 8 + 8
    dx = torch.full((T, ld), 7.0, dtype=dtype, device="cuda")
    dw = torch.full((N, ld), 7.0, device="cuda")
    tng.linear8_grad(dy, x, wt, swt, draw=d, dx=dx[:, :K], dw=dw[:, :K])
    assert torch.equal(dx[:, :K], wanted(*tng.quant8_rows(dy, d), wt, swt, dtype)) and bool((dx[:, K:] == 7).all())
    assert torch.equal(dw[:, :K], wanted(*tng.quant8_cols(dy, d), *tng.quant8_cols(x), torch.float32)) and bool((dw[:, K:] == 7).all())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T,K,N", [(2048, 512, 520), (300, 2600, 2600), (1500, 5000, 20000), (9000, 768, 2900)])
def test_drawn_gradients_of_many_tiles(dtype, T, K, N):
    x, dy = values((T, K), dtype, 1), values((T, N), dtype, 2, 1e-2)
    wt, swt = tng.quant8_cols(values((N, K), torch.float32, 3, K ** -0.5))
    d = tng.Draw(SEED, 4, 8, row0=5)
    dx, dw, _ = tng.linear8_grad(dy, x, wt, swt, draw=d)
    assert torch.equal(dx, wanted(*tng.quant8_rows(dy, d), wt, swt, dtype))
    assert torch.equal(dw, wanted(*tng.quant8_cols(dy, d), *tng.quant8_cols(x), torch.float32))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("drawn", [False, True])
def test_gradients_of_lines_that_are_zero_tiny_or_not_finite(dtype, drawn):
    """dy's row and column codes come from one pass: each line's fate is its own, as when the quantisers code it apart."""
    T, K, N = 300, 40, 200
    clean = values((T, N), dtype, 3)
    x = values((T, K), dtype, 4)
    wt, swt = tng.quant8_cols(values((N, K), torch.float32, 5))
    d = tng.Draw(SEED, 6, 7) if drawn else None
    u = ref.uniforms(T, N, SEED, 6, 7, ref.TAG_ROUNDING) if drawn else None
    tiny = 2.0 ** -126 if dtype != torch.float16 else 2.0 ** -24
    for name, spoil in {"nan": lambda y: y[5, 7].fill_(float("nan")), "inf": lambda y: y[129, 65].fill_(float("inf")),
                        "-inf": lambda y: y[299, 199].fill_(float("-inf")), "rows": lambda y: y[10:20].zero_(), "columns": lambda y: y[:, 60:70].zero_(),
                        "tiny row": lambda y: y[250].mul_(tiny), "tiny column": lambda y: y[:, 130].mul_(tiny),
                        "largest": lambda y: y[77].fill_(torch.finfo(dtype).max)}.items():
        dy = clean.clone()
        spoil(dy)
        dx, dw, db = tng.linear8_grad(dy, x, wt, swt, draw=d)
        wdx, wdw, _ = ref.linear_grad(f32(dy), f32(x), to_np(wt), to_np(swt), u)
        assert same(f32(dx), rounded(wdx, dtype)), name
        assert same(to_np(dw), wdw), name
        row_bad, col_bad = ~torch.isfinite(dy).all(1), ~torch.isfinite(dy).all(0)
        assert torch.equal(torch.isnan(dx).all(1), row_bad) and torch.equal(torch.isnan(dw).all(1), col_bad)
        assert torch.equal(~torch.isfinite(db), col_bad)


@pytest.mark.parametrize("drawn", [False, True])
def test_gradients_can_be_captured_in_a_graph(drawn):
    T, K, N = 300, 512, 260
    x, dy = values((T, K), torch.bfloat16, 1), values((T, N), torch.bfloat16, 2)
    wt, swt = tng.quant8_cols(values((N, K), torch.float32, 3))
    d = tng.Draw(1, 2, 3) if drawn else None
    dx, dw, db = torch.empty_like(x), torch.empty((N, K), device="cuda"), torch.empty(N, device="cuda")
    q, s, sums = tng.empty_codes(K, T), torch.empty(K, device="cuda"), torch.empty(K, device="cuda")
    scratch = torch.empty(tng.lib().tng_linear8_grad_scratch_bytes(T, K, N), dtype=torch.uint8, device="cuda")
    scratch2 = torch.empty(tng.lib().tng_quant8_cols_scratch_bytes(T, K), dtype=torch.uint8, device="cuda")

    def step():
        tng.linear8_grad(dy, x, wt, swt, draw=d, dx=dx, dw=dw, db=db, scratch=scratch)
        tng.quant8_cols(dx, d, q=q, scale=s, colsum=sums, scratch=scratch2)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
        step()                                              # a clear right after a product
    for seed in (5, 6, 7):
        dy.copy_(values((T, N), torch.bfloat16, seed))
        x.copy_(values((T, K), torch.bfloat16, seed + 10))
        graph.replay()
        got = [t.clone() for t in (dx, dw, db, q, s, sums)]
        step()
        assert all(torch.equal(a, b) for a, b in zip(got, (dx, dw, db, q, s, sums)))
        assert torch.equal(dx, tng.linear8_grad(dy, x, wt, swt, draw=d)[0])


@pytest.mark.parametrize("dtype,cols", [(torch.float32, 40007), (torch.bfloat16, 70001), (torch.float16, 131056), (torch.float32, 131056)])
def test_rows_longer_than_a_block_holds(dtype, cols):
    """Rows that the registers of 1024 threads do not hold are read a second time."""
    x = values((3, cols), dtype, 1)
    x[1, cols - 1] = 50.0                                   # the largest lies in the part that is not kept
    for draw in (None, tng.Draw(SEED, 5, 77, row0=3)):
        u = None if draw is None else ref.uniforms(3, cols, SEED, 5, 77, ref.TAG_ROUNDING, 3)
        q, s = tng.quant8_rows(x, draw)
        wq, ws = ref.codes(f32(x), u)
        assert same(to_np(q), wq) and same(to_np(s), ws)


@pytest.mark.parametrize("n", [264, 261])
def test_products_of_rows_far_apart(n):
    """Codes and outputs whose last rows lie beyond 32 bits of bytes: tiled copies and scalar stores."""
    m, k = 130, 200
    a, sa = random_codes(m, k, 1)
    b, sb = random_codes(n, k, 2)
    want = wanted(a, sa, b, sb, torch.bfloat16)
    ld = (1 << 25) + 64
    far = torch.empty((m - 1) * ld + 256, dtype=torch.int8, device="cuda").as_strided((m, k), (ld, 1))
    far.copy_(a)
    out = torch.empty((m - 1) * ld + 512, dtype=torch.bfloat16, device="cuda").as_strided((m, n), (ld, 1))
    tng.product8(far, sa, b, sb, out=out)
    assert torch.equal(out, want)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T", [1, 5, 8, 12, 70])
def test_what_follows_a_line_does_not_count(dtype, T):
    """Weights that are a part of wider codes, activations and outputs that are parts of wider rows."""
    K, N = 203, 37
    wide, sw = random_codes(N, K + 45, 1)
    x = torch.full((T, K + 5), float("nan"), dtype=dtype, device="cuda")
    x[:, :K] = values((T, K), dtype, 2)
    y = torch.full((T, N + 3), 7.0, dtype=dtype, device="cuda")
    tng.linear8(x[:, :K], wide[:, :K], sw, out=y[:, :N])
    want = ref.linear(f32(x[:, :K]), to_np(wide[:, :K]), to_np(sw))
    assert same(f32(y[:, :N]), rounded(want, dtype)) and bool((y[:, N:] == 7).all())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols", [(3, 5), (40, 1000), (300, 4097), (2000, 1030)])
def test_dropout_writes_its_columns_only(dtype, rows, cols):
    x = values((rows, cols), dtype, 1)
    d = tng.Draw(SEED, 3, 12)
    want = tng.dropout(x, 0.3, d, residual=x)
    for ld in (cols + 1, -(-cols // 8) * 8 + 8):
        base = torch.full((rows + 1, ld), 7.0, dtype=dtype, device="cuda")
        tng.dropout(x, 0.3, d, residual=x, out=base[:rows, :cols])
        assert torch.equal(base[:rows, :cols], want) and bool((base[:rows, cols:] == 7).all()) and bool((base[rows] == 7).all())
