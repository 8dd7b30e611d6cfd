"""Layer operators at the edges of their tiles, launches and buffers (see test_gpu_layers.py for the operators themselves)."""
import pytest
import torch

from paper_1901_08227_b200 import tng
from test_gpu_layers import DTYPES, SEED, random_codes, values

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
