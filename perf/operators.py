"""Workloads of the training-layer operators: 8-bit linear layers (forward and gradient) and counter-based dropout.

``own`` chooses between the plain form of an operator (elementary torch operations in 32 bits, one rounding at the
end) and the library's calls; both take the same state and return outputs of the same layout.

Definitions.  A line (a row for a scale per token, a column for a scale per channel) with A = max|x| is held as codes
q and a scale: scale = A/127, inv = 127/A, v = x inv, each one fp32 operation; q = rint(v), half to even, or, with a
draw, q = floor(v + u) cut to [-127, 127] (the sum one fp32 operation, u a 24-bit uniform).  A line that is zero (A below
2^-120) has scale 0 and codes 0.  Uniforms are Philox4x32-10 with the seed as key and the counter
(column // 4, row, layer + tag, step); word column % 4 belongs to the column; tag 2^30 for rounding, 2^31 for dropout.
"""
import math

import torch

own = False

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
SIZE = {"fp32": 4, "bf16": 2, "fp16": 2}
ROUNDING, DROPOUT = 1 << 30, 1 << 31
TINY = 2.0 ** -120
MOST_FLOPS = 2 * 8192 ** 3          # the largest listed product; drawn ones stay below
MOST_ELEMENTS = 16384 * 8192        # the largest listed dropout


def listed():
    return [
        # one token through a square projection: the decode step of serving, all latency and weight traffic
        {"name": "linear8 one token", "op": "linear", "dtype": "bf16", "T": 1, "K": 4096, "N": 4096, "bias": False},
        # a few requests decoded together, wide output layer, half precision with a bias
        {"name": "linear8 eight tokens", "op": "linear", "dtype": "fp16", "T": 8, "K": 2048, "N": 16384, "bias": True},
        # a short prompt: too few tokens to fill the GPU by rows alone
        {"name": "linear8 prompt", "op": "linear", "dtype": "bf16", "T": 512, "K": 4096, "N": 4096, "bias": True},
        # sizes that are multiples of nothing, full-precision activations
        {"name": "linear8 ragged", "op": "linear", "dtype": "fp32", "T": 1333, "K": 1001, "N": 2503, "bias": True},
        # a training batch through a wide layer: bound by the matrix unit
        {"name": "linear8 batch", "op": "linear", "dtype": "bf16", "T": 8192, "K": 8192, "N": 8192, "bias": False},
        # gradients of a small layer at odd sizes, as in the tests of a new model, fp32 throughout
        {"name": "linear8 grad ragged", "op": "linear_grad", "dtype": "fp32", "T": 777, "K": 1000, "N": 515, "draw": False},
        # gradients of one worker's micro-batch, gradient rounded without bias
        {"name": "linear8 grad worker", "op": "linear_grad", "dtype": "bf16", "T": 2048, "K": 4096, "N": 4096, "draw": True},
        # gradients of a large batch through a square layer
        {"name": "linear8 grad batch", "op": "linear_grad", "dtype": "bf16", "T": 16384, "K": 4096, "N": 4096, "draw": False},
        # dropout and residual sum of a handful of tokens: latency
        {"name": "dropout few", "op": "dropout", "dtype": "bf16", "rows": 16, "cols": 1024, "p": 0.1, "residual": True},
        # dropout and residual sum of a training batch
        {"name": "dropout batch", "op": "dropout", "dtype": "bf16", "rows": 16384, "cols": 8192, "p": 0.1, "residual": True},
        # its gradient at odd sizes (rows that start anywhere), fp32
        {"name": "dropout grad ragged", "op": "dropout_grad", "dtype": "fp32", "rows": 4097, "cols": 2501, "p": 0.5},
        # its gradient for a training batch
        {"name": "dropout grad batch", "op": "dropout_grad", "dtype": "fp16", "rows": 8192, "cols": 8192, "p": 0.25},
    ]


def draw(rng):
    def size(lo, hi):
        n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
        if rng.random() < 0.5 and n >= 64:
            n -= n % 64
        return max(lo, min(hi, n))

    op = rng.choice(["linear", "linear", "linear_grad", "linear_grad", "dropout", "dropout_grad"])
    dtype = rng.choice(["bf16", "bf16", "fp16", "fp32"])
    while op == "linear":
        c = {"op": op, "dtype": dtype, "T": size(1, 16384), "K": size(128, 16384), "N": size(128, 16384), "bias": rng.random() < 0.5}
        if 2 * c["T"] * c["K"] * c["N"] <= MOST_FLOPS:
            return c
    while op == "linear_grad":
        c = {"op": op, "dtype": dtype, "T": size(1, 16384), "K": size(128, 16384), "N": size(128, 16384), "draw": rng.random() < 0.5}
        if 4 * c["T"] * c["K"] * c["N"] <= MOST_FLOPS:
            return c
    while True:
        c = {"op": op, "dtype": dtype, "rows": size(1, 32768), "cols": size(128, 16384), "p": rng.choice([0.05, 0.1, 0.25, 0.5])}
        if op == "dropout":
            c["residual"] = rng.random() < 0.7
        if c["rows"] * c["cols"] <= MOST_ELEMENTS:
            return c


def _line_codes(w):
    """Weights (n, k) in 32 bits -> codes whose rows start on 16-byte boundaries, one scale a row."""
    n, k = w.shape
    a = w.abs().amax(1)
    q = torch.zeros((n, -(-k // 16) * 16), dtype=torch.int8, device=w.device)
    q[:, :k] = torch.round(w * (127.0 / a)[:, None]).to(torch.int8)
    return q[:, :k], a / 127.0


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dt = DTYPES[case["dtype"]]

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    s = {"case": dict(case), "seed": 0x1234567800000000 + seed % (1 << 31), "layer": seed % 64, "step": seed % 10007}
    if case["op"] in ("dropout", "dropout_grad"):
        rows, cols = case["rows"], case["cols"]
        if case["op"] == "dropout":
            s["x"] = normal(rows, cols).to(dt)
            s["residual"] = normal(rows, cols).to(dt) if case["residual"] else None
        else:
            s["dy"] = (1e-3 * normal(rows, cols)).to(dt)
        return s
    T, K, N = case["T"], case["K"], case["N"]
    # activations: a few channels are much larger than the rest
    x = normal(T, K)
    x *= 1.0 + 15.0 * (torch.rand((1, K), generator=g, device="cuda") < 0.01)
    s["x"] = x.to(dt)
    del x
    w = normal(N, K) / math.sqrt(K)
    if case["op"] == "linear":
        s["wq"], s["ws"] = _line_codes(w)                       # a scale an output channel
        s["bias"] = 0.1 * normal(N) if case["bias"] else None
    else:
        s["wt"], s["wts"] = _line_codes(w.t().contiguous())     # a scale an input channel
        dy = 1e-3 * normal(T, N) * torch.exp(normal(T, 1))      # tokens differ in size
        dy[torch.rand(T, generator=g, device="cuda") < 0.1] = 0.0   # padding: no gradient at all
        s["dy"] = dy.to(dt)
    return s


# ---- plain forms ---------------------------------------------------------------------------------

def _words(rows, cols, seed, word2, step, device):
    """The 32-bit Philox words of a (rows, cols) array, as int64."""
    m = 0xFFFFFFFF
    n4 = -(-cols // 4)
    c0 = torch.arange(n4, device=device).expand(rows, n4)
    c1 = torch.arange(rows, device=device)[:, None].expand(rows, n4)
    c2 = torch.full_like(c0, word2)
    c3 = torch.full_like(c0, step)
    k0, k1 = seed & m, (seed >> 32) & m
    for _ in range(10):
        p0, p1 = c0 * 0xD2511F53, c2 * 0xCD9E8D57      # 64-bit products, wrapped into int64
        c0, c1, c2, c3 = ((p1 >> 32) & m) ^ c1 ^ k0, p1 & m, ((p0 >> 32) & m) ^ c3 ^ k1, p0 & m
        k0, k1 = (k0 + 0x9E3779B9) & m, (k1 + 0xBB67AE85) & m
    return torch.stack((c0, c1, c2, c3), dim=-1).reshape(rows, 4 * n4)[:, :cols]


def _uniforms(*a):
    return (_words(*a) >> 8).float() * 2.0 ** -24


def _codes(x, dim, u=None):
    """x in 32 bits -> codes (as fp32 numbers) and scales along `dim`."""
    a = x.abs().amax(dim, keepdim=True)
    zero = a < TINY
    top = torch.full_like(a, 127.0)             # a tensor: torch multiplies by a scalar's rounded reciprocal instead of dividing
    inv = torch.where(zero, torch.zeros_like(a), top / a)
    v = x * inv
    q = torch.round(v) if u is None else torch.floor(v + u).clamp(-127.0, 127.0)
    return torch.where(zero, torch.zeros_like(q), q), torch.where(zero, torch.zeros_like(a), a / top)


def _dropped(x, p, s):
    u = _uniforms(x.shape[0], x.shape[1], s["seed"], s["layer"] + DROPOUT, s["step"], x.device)
    keep = 1.0 / (1.0 - torch.tensor(p))                       # in fp32, once
    return torch.where(u >= p, x.float() * float(keep), torch.zeros((), device=x.device))


def _plain(s):
    c = s["case"]
    if c["op"] == "dropout":
        y = _dropped(s["x"], c["p"], s)
        return (y if s["residual"] is None else s["residual"].float() + y).to(s["x"].dtype)
    if c["op"] == "dropout_grad":
        return _dropped(s["dy"], c["p"], s).to(s["dy"].dtype)
    if c["op"] == "linear":
        q, sx = _codes(s["x"].float(), 1)
        y = torch.matmul(q, s["wq"].float().t()) * sx * s["ws"]
        return (y if s["bias"] is None else y + s["bias"]).to(s["x"].dtype)
    dy = s["dy"].float()
    u = _uniforms(dy.shape[0], dy.shape[1], s["seed"], s["layer"] + ROUNDING, s["step"], dy.device) if c["draw"] else None
    qr, sr = _codes(dy, 1, u)
    dx = torch.matmul(qr, s["wt"].float().t()) * sr * s["wts"]
    qc, sc = _codes(dy, 0, u)
    qx, sx = _codes(s["x"].float(), 0)
    dw = torch.matmul(qc.t(), qx) * sc.t() * sx
    return {"dx": dx.to(s["dy"].dtype), "dw": dw, "db": dy.sum(0)}


# ---- the library's calls -------------------------------------------------------------------------

def _own(s):
    from paper_1901_08227_b200 import tng

    c = s["case"]
    if c["op"] == "linear":
        return tng.linear8(s["x"], s["wq"], s["ws"], bias=s["bias"])
    if c["op"] == "linear_grad":
        d = tng.Draw(s["seed"], s["layer"], s["step"]) if c["draw"] else None
        dx, dw, db = tng.linear8_grad(s["dy"], s["x"], s["wt"], s["wts"], draw=d)
        return {"dx": dx, "dw": dw, "db": db}
    d = tng.Draw(s["seed"], s["layer"], s["step"])
    if c["op"] == "dropout":
        return tng.dropout(s["x"], c["p"], d, residual=s["residual"])
    return tng.dropout_grad(s["dy"], c["p"], d)


def run(state):
    return _own(state) if own else _plain(state)


def work(case):
    e = SIZE[case["dtype"]]
    if case["op"] in ("dropout", "dropout_grad"):
        n = case["rows"] * case["cols"]
        return {"bytes": e * n * (3 if case.get("residual") else 2), "flops": 2 * n}
    T, K, N = case["T"], case["K"], case["N"]
    if case["op"] == "linear":
        return {"bytes": e * T * K + N * K + 4 * N + e * T * N + (4 * N if case["bias"] else 0), "flops": 2 * T * K * N}
    return {"bytes": e * T * N + e * T * K + K * N + 4 * K + e * T * K + 4 * N * K + 4 * N, "flops": 4 * T * K * N}


# ---- the definitions in 64 bits ------------------------------------------------------------------

def _exact_words(row, n4, seed, word2, step):
    """Philox words of rows `row` (a vector), four a counter; products by 16-bit limbs."""
    def mul(a, k):                                       # a, k < 2^32 -> high and low word
        lo = a * (k & 0xFFFF)
        hi = a * (k >> 16)
        low = lo + ((hi & 0xFFFF) << 16)
        return (hi >> 16) + (low >> 32), low & 0xFFFFFFFF

    block = [torch.arange(n4, device="cuda")[None, :] + 0 * row[:, None], row[:, None] + torch.zeros(n4, dtype=torch.int64, device="cuda")]
    block += [torch.zeros_like(block[0]) + word2, torch.zeros_like(block[0]) + step]
    for r in range(10):
        key = [((seed & 0xFFFFFFFF) + r * 0x9E3779B9) % (1 << 32), ((seed >> 32) + r * 0xBB67AE85) % (1 << 32)]
        h0, l0 = mul(block[0], 0xD2511F53)
        h1, l1 = mul(block[2], 0xCD9E8D57)
        block = [h1 ^ block[1] ^ key[0], l1, h0 ^ block[3] ^ key[1], l0]
    return torch.stack(block, 2).flatten(1)


def _exact_uniforms(rows, cols, seed, word2, step):
    out = torch.empty((rows, cols), dtype=torch.float64, device="cuda")
    per = max(1, (1 << 24) // cols)
    for r0 in range(0, rows, per):
        r1 = min(rows, r0 + per)
        w = _exact_words(torch.arange(r0, r1, device="cuda"), (cols + 3) // 4, seed, word2, step)
        out[r0:r1] = torch.div(w[:, :cols], 256, rounding_mode="floor").double() / 2.0 ** 24
    return out


def _exact_codes(x, u=None):
    """Lines are the rows of x (64 bits).  The fp32 operations that decide a code are part of its definition: each is the
    64-bit result rounded to fp32 (exact products; quotients and sums of fp32 numbers round the same way)."""
    def single(v):
        return v.to(torch.float32).to(torch.float64)

    a = x.abs().max(dim=1, keepdim=True).values
    live = a >= TINY
    safe = torch.where(live, a, torch.ones_like(a))
    v = single(x * single(127.0 / safe))
    q = v.round() if u is None else single(v + u).floor().clamp(-127, 127)
    return q * live, single(safe / 127.0) * live


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] in ("dropout", "dropout_grad"):
        x = s["x"] if case["op"] == "dropout" else s["dy"]
        u = _exact_uniforms(x.shape[0], x.shape[1], s["seed"], s["layer"] + DROPOUT, s["step"])
        y = torch.where(u < case["p"], 0.0, x.double() / (1.0 - case["p"]))
        return y + s["residual"].double() if case.get("residual") else y
    if case["op"] == "linear":
        q, sx = _exact_codes(s["x"].double())
        y = (q @ s["wq"].double().T) * (sx * s["ws"].double()[None, :])
        return y if s["bias"] is None else y + s["bias"].double()[None, :]
    dy, x = s["dy"].double(), s["x"].double()
    u = _exact_uniforms(dy.shape[0], dy.shape[1], s["seed"], s["layer"] + ROUNDING, s["step"]) if case["draw"] else None
    q, sr = _exact_codes(dy, u)
    dx = (q @ s["wt"].double().T) * (sr * s["wts"].double()[None, :])
    q, sc = _exact_codes(dy.T, None if u is None else u.T)
    qx, sx = _exact_codes(x.T)
    return {"dx": dx, "dw": (q @ qx.T) * (sc * sx.T), "db": dy.sum(dim=0)}
