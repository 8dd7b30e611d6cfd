"""What the calls of the token operators refuse, and what the binding passes on (CPU only: no call here reaches a GPU)."""
import ctypes as C

import pytest
import torch

from paper_1901_08227_b200 import tng

BF16, F32 = tng.BF16, tng.F32
P = 1 << 20                                                 # an address that nobody follows: every call is refused before
BIG = 1 << 31


def embed(table=P, tt=BF16, vocab=10, width=32, ldt=32, ids=P, id_bytes=8, tokens=4, y=P, type=BF16, ldy=32):
    return tng.lib().tng_embed(table, tt, vocab, width, ldt, ids, id_bytes, tokens, 1.0, y, type, ldy, None)


def embed_grad(dy=P, type=BF16, tokens=4, width=32, lddy=32, ids=P, id_bytes=8, vocab=10, dtable=P, ldd=32, scratch=P):
    return tng.lib().tng_embed_grad(dy, type, tokens, width, lddy, ids, id_bytes, vocab, 1.0, dtable, ldd, scratch, None)


def rmsnorm(x=P, type=BF16, rows=4, cols=32, ldx=32, res=None, ldres=0, w=P, eps=1e-6, h=None, ldh=0, y=P, ldy=32, q=None, ldq=0, scale=None, r=None):
    return tng.lib().tng_rmsnorm(x, type, rows, cols, ldx, res, ldres, w, eps, h, ldh, y, ldy, q, ldq, scale, r, None)


def rmsnorm_grad(dy=P, lddy=32, h=P, ldh=32, type=BF16, rows=4, cols=32, w=P, r=P, dres=None, lddres=0, dx=P, lddx=32, dw=P, scratch=P):
    return tng.lib().tng_rmsnorm_grad(dy, lddy, h, ldh, type, rows, cols, w, r, dres, lddres, dx, lddx, dw, scratch, None)


def orthogonalize(v=P, type=F32, batch=1, rows=8, cols=16, ldv=16, stride=0, steps=5, a=3.4445, b=-4.775, c=2.0315, out=P, ot=F32, ldo=16, ostride=0, scratch=P):
    return tng.lib().tng_orthogonalize(v, type, batch, rows, cols, ldv, stride, steps, a, b, c, out, ot, ldo, ostride, scratch, None)


NAN, INF = float("nan"), float("inf")
REFUSED = [(embed, k) for k in [dict(table=None), dict(ids=None), dict(y=None), dict(tt=3), dict(type=-1), dict(id_bytes=2), dict(id_bytes=0), dict(vocab=0), dict(width=0),
                                dict(ldt=31), dict(ldy=31), dict(table=P + 1), dict(y=P + 1), dict(ids=P + 4), dict(ids=P + 2, id_bytes=4), dict(vocab=BIG), dict(tokens=BIG),
                                dict(width=BIG, ldt=BIG, ldy=BIG)]]
REFUSED += [(embed_grad, k) for k in [dict(dy=None), dict(ids=None), dict(dtable=None), dict(scratch=None), dict(scratch=P + 128), dict(type=7), dict(id_bytes=16), dict(vocab=0),
                                      dict(width=0), dict(lddy=31), dict(ldd=31), dict(dtable=P + 2), dict(dy=P + 1), dict(ids=P + 4), dict(vocab=BIG), dict(tokens=BIG),
                                      dict(width=(1 << 26) + 1, lddy=1 << 27, ldd=1 << 27)]]
REFUSED += [(rmsnorm, k) for k in [dict(x=None), dict(w=None), dict(type=3), dict(cols=0), dict(ldx=31), dict(ldy=31), dict(x=P + 1), dict(w=P + 2), dict(r=P + 2), dict(eps=0.0),
                                   dict(eps=-1e-6), dict(eps=NAN), dict(eps=INF), dict(eps=1e-40), dict(res=P, ldres=31), dict(res=P + 1, ldres=32), dict(h=P, ldh=31),
                                   dict(h=P + 1, ldh=32), dict(q=P, ldq=32), dict(q=P, ldq=31, scale=P), dict(q=P, ldq=40, scale=P), dict(q=P + 8, ldq=32, scale=P),
                                   dict(q=P, ldq=32, scale=P + 2), dict(rows=BIG), dict(cols=BIG, ldx=BIG, ldy=BIG)]]
REFUSED += [(rmsnorm_grad, k) for k in [dict(dy=None), dict(h=None), dict(w=None), dict(r=None), dict(scratch=None), dict(scratch=P + 16), dict(type=5), dict(cols=0), dict(lddy=31),
                                        dict(ldh=31), dict(lddx=31), dict(dres=P, lddres=31), dict(dres=P + 1, lddres=32), dict(dy=P + 1), dict(dx=P + 1), dict(dw=P + 2), dict(rows=BIG)]]
REFUSED += [(orthogonalize, k) for k in [dict(v=None), dict(out=None), dict(scratch=None), dict(scratch=P + 64), dict(type=4), dict(ot=4), dict(rows=0), dict(cols=0), dict(ldv=15),
                                         dict(ldo=15), dict(v=P + 2), dict(out=P + 2), dict(steps=0), dict(steps=65), dict(batch=65536), dict(batch=2), dict(a=NAN), dict(b=INF),
                                         dict(c=-INF), dict(a=2.5, b=0.0, c=0.0), dict(a=16.0, b=-60.0, c=50.0), dict(a=1.9, b=0.9, c=0.0, steps=2), dict(rows=1 << 30, cols=1, ldv=1, ldo=1),
                                         dict(batch=60000, rows=65536, cols=16, stride=1 << 20, ostride=1 << 20)]]


@pytest.mark.parametrize("call,change", REFUSED, ids=lambda v: v.__name__ if callable(v) else ",".join(v))
def test_calls_are_refused_before_they_reach_the_device(call, change):
    assert call(**change) == tng.ERR_INVALID_ARG


def test_nothing_to_do_succeeds_without_a_device():
    assert embed(tokens=0) == tng.OK
    assert rmsnorm(rows=0) == tng.OK
    assert rmsnorm_grad(rows=0, dw=None) == tng.OK
    assert rmsnorm_grad(dx=None, dw=None) == tng.OK
    assert orthogonalize(batch=0) == tng.OK


def test_scratch_sizes():
    L = tng.lib()
    assert L.tng_embed_grad_scratch_bytes(0, 100) >= 1 and L.tng_rmsnorm_grad_scratch_bytes(0, 100) >= 1 and L.tng_orthogonalize_scratch_bytes(0, 8, 8) >= 1
    for tokens in (1, 100, 1 << 20, BIG - 1):
        assert 16 * tokens < L.tng_embed_grad_scratch_bytes(tokens, 64) < 16 * tokens + (64 + 64 * 8) * 8193 + 4096
    assert L.tng_rmsnorm_grad_scratch_bytes(BIG - 1, 4096) <= 148 * 4 * 4096 * 4
    for m, n in ((1, 1), (515, 1001), (4096, 4096)):
        assert L.tng_orthogonalize_scratch_bytes(3, m, n) == L.tng_orthogonalize_scratch_bytes(3, n, m) >= 3 * 4 * (3 * m * n + 2 * min(m, n) ** 2)


class Recorder:
    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            self.calls.append((name, args))
            return 256 if name.endswith("_bytes") else tng.OK
        return call


@pytest.fixture
def library(monkeypatch):
    r = Recorder()
    monkeypatch.setattr(tng, "lib", lambda: r)
    monkeypatch.setattr(tng, "_device", lambda t=None: -1)      # what get_device() says of a CPU tensor
    monkeypatch.setattr(tng, "_stream", lambda dev=None: 0)
    monkeypatch.setattr(tng, "_scratch", lambda *a: (None, None))
    return r


def args_of(library, name):
    (args,) = [a for n, a in library.calls if n == name]
    return args


def test_strides_types_and_sizes_are_passed_on(library):
    table = torch.zeros((7, 40))[:, :33]
    ids = torch.zeros(5, dtype=torch.int32)
    out = tng.embed(table, ids, scale=2.0, dtype=torch.bfloat16)
    a = args_of(library, "tng_embed")
    assert a[1:5] == (F32, 7, 33, 40) and a[6:9] == (4, 5, 2.0) and a[9:12] == (out.data_ptr(), BF16, 33)
    row = torch.zeros(1000)
    d = tng.embed_grad(torch.zeros((5, 33)), ids, 7, dtable=row[11:11 + 7 * 33].view(7, 33))
    a = args_of(library, "tng_embed_grad")
    assert a[8:11] == (1.0, row.data_ptr() + 44, 33) and d.data_ptr() == row.data_ptr() + 44
    x = torch.zeros((3, 48), dtype=torch.float16)[:, :20]
    q, s, h, r = tng.rmsnorm8(x, torch.zeros(20), residual=torch.zeros((3, 20), dtype=torch.float16))
    a = args_of(library, "tng_rmsnorm")
    assert a[1:5] == (tng.F16, 3, 20, 48) and a[6] == 20 and a[13:15] == (q.data_ptr(), 32) and h.shape == (3, 20) and q.shape == (3, 20) and q.stride(0) == 32
    assert s.dtype == r.dtype == torch.float32
    v = torch.zeros((4, 3, 10, 20)).permute(1, 0, 2, 3)[0]      # three layers' matrices side by side
    tng.orthogonalize(v)
    a = args_of(library, "tng_orthogonalize")
    assert a[2:8] == (4, 10, 20, 20, 600, 5) and a[13:15] == (20, 200)


@pytest.mark.parametrize("default", [torch.float64, torch.bfloat16])
def test_new_outputs_do_not_follow_the_default_type(library, default):
    before = torch.get_default_dtype()
    torch.set_default_dtype(default)
    try:
        x, w = torch.zeros((3, 20), dtype=torch.float32), torch.ones(20, dtype=torch.float32)
        q, s, h, r = tng.rmsnorm8(x, w)
        assert s.dtype == r.dtype == torch.float32 and q.dtype == torch.int8
        assert tng.rmsnorm_grad(x.half(), x.half(), w, r)[1].dtype == torch.float32
        assert tng.embed_grad(x.half(), torch.zeros(3, dtype=torch.int64), 4).dtype == torch.float32
        assert tng.orthogonalize(x).dtype == torch.float32
    finally:
        torch.set_default_dtype(before)


def test_codes_without_their_padding_are_refused(library):
    pool = torch.zeros(64, dtype=torch.int8)
    with pytest.raises(ValueError):
        tng.rmsnorm8(torch.zeros((1, 20)), torch.ones(20), q=pool[:20].view(1, 20))


def test_weights_are_not_optional(library):
    x = torch.zeros((3, 20))
    with pytest.raises(TypeError):
        tng.rmsnorm(x, None)
    with pytest.raises(TypeError):
        tng.rmsnorm8(x, None)
