"""Workloads of the operators around the 8-bit layers of a token model: embedding rows and their gradient, root-mean-square norm
with the residual's addition and 8-bit codes, its gradient, and the orthogonalised update of weight matrices.

``own`` chooses between the plain form of an operator (elementary torch operations in 32 bits, one rounding at the end) and
the library's calls; both take the same state and return outputs of the same layout.

Definitions.
  embed       y[t] = table[ids[t]] scale (an fp32 product, rounded to y's type); an id of -1 is an empty place: a row of zeros.
  embed_grad  dtable[v] = scale * sum of dy[t] over the t with ids[t] = v: fp32, every row written.
  norm        h = x + residual rounded to the type (one fp32 sum), r = 1 / sqrt(mean of h^2 + eps), and either y = h r w in the
              type or codes of y by row.  The codes do not depend on r: with t = h w (one fp32 product) and A = max|t|,
              inv = 127/A, q = rint(t inv), half to even, and the scale is (A/127) r.
  norm_grad   g = dy w, dx = r (g - h r^2 mean(g h)) + dres in the type, dw = sum over the rows of dy h r in fp32.
  orthogonal  X = V / |V| in Frobenius norm, then `steps` times X <- (a I + b G + c G^2) X with G = X X^T, for every matrix of
              a batch: all singular values move towards one.  (On the shorter side, whichever it is: the result is the same.)
"""
import math

import torch

own = False

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
SIZE = {"fp32": 4, "bf16": 2, "fp16": 2}
EPS = 1e-6
COEFFICIENTS = (3.4445, -4.7750, 2.0315)
MOST_TABLE = 65536 * 2048            # elements of the largest listed table, of its batch, of the largest listed norm, and the
MOST_TOKENS = 32768 * 2048           # products of the largest listed update; drawn cases stay below
MOST_NORM = 16384 * 8192
MOST_UPDATE = 5 * (3 * 4096 * 4096 * 16384 + 4096 ** 3)


def listed():
    return [
        # the row of the token that serving decodes next: all latency
        {"name": "embed one token", "op": "embed", "dtype": "bf16", "table": "bf16", "T": 1, "V": 32768, "k": 4096, "scale": 1.0},
        # a training batch from full-precision weights, scaled by the root of the width; a part of the places is padding
        {"name": "embed batch", "op": "embed", "dtype": "bf16", "table": "fp32", "T": 16384, "V": 65536, "k": 2048, "scale": 45.25},
        # gradients of a small vocabulary at sizes that are multiples of nothing, fp32 throughout, as in tests of a new model
        {"name": "embed grad ragged", "op": "embed_grad", "dtype": "fp32", "T": 1777, "V": 10007, "k": 515, "scale": 1.0},
        # gradients of a training batch: many tokens share a few ids
        {"name": "embed grad batch", "op": "embed_grad", "dtype": "bf16", "T": 32768, "V": 65536, "k": 2048, "scale": 45.25},
        # one token on its way into an 8-bit layer: the decode step of serving, all latency
        {"name": "norm one token", "op": "norm", "dtype": "bf16", "T": 1, "k": 4096, "residual": True, "codes": True},
        # rows that start anywhere, full precision, no codes
        {"name": "norm ragged", "op": "norm", "dtype": "fp32", "T": 1333, "k": 1001, "residual": True, "codes": False},
        # a training batch into an 8-bit layer
        {"name": "norm batch", "op": "norm", "dtype": "bf16", "T": 16384, "k": 8192, "residual": True, "codes": True},
        # gradients at odd sizes, half precision
        {"name": "norm grad ragged", "op": "norm_grad", "dtype": "fp16", "T": 777, "k": 1001, "dres": False},
        # gradients of a training batch, the residual's gradient added on the way
        {"name": "norm grad batch", "op": "norm_grad", "dtype": "bf16", "T": 16384, "k": 4096, "dres": True},
        # the update of one small square layer: a chain of short products
        {"name": "orthogonal small", "op": "orthogonal", "dtype": "bf16", "batch": 1, "m": 512, "n": 512, "steps": 5},
        # odd sizes, taller than wide, three layers of a shape at once, straight from the fp32 aggregate of a round
        {"name": "orthogonal ragged", "op": "orthogonal", "dtype": "fp32", "batch": 3, "m": 1001, "n": 515, "steps": 5},
        # a wide layer's aggregate: bound by the matrix unit
        {"name": "orthogonal wide", "op": "orthogonal", "dtype": "fp32", "batch": 1, "m": 4096, "n": 16384, "steps": 5},
    ]


def draw(rng):
    def size(lo, hi):
        n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
        if rng.random() < 0.5 and n >= 64:
            n -= n % 64
        return max(lo, min(hi, n))

    op = rng.choice(["embed", "embed_grad", "embed_grad", "norm", "norm", "norm_grad", "orthogonal", "orthogonal"])
    dtype = rng.choice(["bf16", "bf16", "fp16", "fp32"])
    while op in ("embed", "embed_grad"):
        c = {"op": op, "dtype": dtype, "T": size(1, 65536), "V": size(128, 131072), "k": size(64, 8192), "scale": rng.choice([1.0, 0.125, 22.6])}
        if op == "embed":
            c["table"] = rng.choice([dtype, "fp32"])
        if c["V"] * c["k"] <= MOST_TABLE and c["T"] * c["k"] <= MOST_TOKENS:
            return c
    while op == "norm":
        c = {"op": op, "dtype": dtype, "T": size(1, 32768), "k": size(64, 16384), "residual": rng.random() < 0.7, "codes": rng.random() < 0.6}
        if c["T"] * c["k"] * SIZE[dtype] <= MOST_NORM * 2:
            return c
    while op == "norm_grad":
        c = {"op": op, "dtype": dtype, "T": size(1, 32768), "k": size(64, 16384), "dres": rng.random() < 0.6}
        if 2 * c["T"] * c["k"] * SIZE[dtype] <= MOST_NORM * 2:
            return c
    while True:
        c = {"op": op, "dtype": dtype, "batch": rng.choice([1, 1, 1, 2, 4]), "m": size(64, 8192), "n": size(64, 16384), "steps": rng.choice([5, 5, 3, 6])}
        if work(c)["flops"] <= MOST_UPDATE:
            return c


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dt = DTYPES[case["dtype"]]

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    s = {"case": dict(case)}
    if case["op"] in ("embed", "embed_grad"):
        T, V, k = case["T"], case["V"], case["k"]
        # ids fall off like 1 / rank, as words do; a few places are padding
        u = torch.rand(T, generator=g, device="cuda", dtype=torch.float64)
        ids = (torch.exp(u * math.log(V + 1.0)) - 1.0).long().clamp(0, V - 1)
        if T > 16:
            ids[torch.rand(T, generator=g, device="cuda") < 0.03] = -1
        s["ids"] = ids
        if case["op"] == "embed":
            s["table"] = (normal(V, k) * k ** -0.5).to(DTYPES[case["table"]])
        else:
            s["dy"] = (1e-3 * normal(T, k) * torch.exp(normal(T, 1))).to(dt)      # tokens differ in size
        return s
    if case["op"] in ("norm", "norm_grad"):
        T, k = case["T"], case["k"]
        s["w"] = 1.0 + 0.1 * normal(k)
        # activations: a few channels are much larger than the rest
        big = 1.0 + 15.0 * (torch.rand((1, k), generator=g, device="cuda") < 0.01)
        if case["op"] == "norm":
            s["x"] = normal(T, k).to(dt)
            s["residual"] = (normal(T, k) * big).to(dt) if case["residual"] else None
        else:
            h = normal(T, k) * big
            s["h"] = h.to(dt)
            s["r"] = torch.rsqrt(s["h"].float().square().mean(1) + EPS)           # kept by the forward pass
            dy = 1e-3 * normal(T, k) * torch.exp(normal(T, 1))
            dy[torch.rand(T, generator=g, device="cuda") < 0.1] = 0.0             # padding: no gradient at all
            s["dy"] = dy.to(dt)
            s["dres"] = (1e-3 * normal(T, k)).to(dt) if case["dres"] else None
        return s
    b, m, n = case["batch"], case["m"], case["n"]
    # an aggregate: a few strong directions over noise
    rank = max(1, min(m, n) // 16)
    v = normal(b, m, n) * 1e-3
    fall = torch.exp(-4.0 * torch.arange(rank, device="cuda") / rank)
    v += 1e-2 * torch.matmul(normal(b, m, rank) * fall, normal(b, rank, n)) / math.sqrt(rank)
    s["v"] = v.to(dt)
    return s


# ---- plain forms ---------------------------------------------------------------------------------

def _rounded_sum(x, residual):
    return x if residual is None else (x.float() + residual.float()).to(x.dtype)


def _plain_norm(s, c):
    h = _rounded_sum(s["x"], s["residual"])
    f = h.float()
    r = 1.0 / torch.sqrt(f.square().mean(1) + EPS)
    out = {"r": r}
    if c["residual"]:
        out["h"] = h
    if not c["codes"]:
        out["y"] = (f * r[:, None] * s["w"]).to(h.dtype)
        return out
    t = f * s["w"]
    top = t.abs().amax(1, keepdim=True)
    full = torch.full_like(top, 127.0)           # a tensor: torch multiplies by a scalar's rounded reciprocal instead of dividing
    out["q"] = torch.round(t * (full / top)).to(torch.int8)
    out["scale"] = (top / full)[:, 0] * r
    return out


def _plain_orthogonal(v, steps):
    a, b, c = COEFFICIENTS
    x = v.float()
    tall = x.shape[1] > x.shape[2]
    if tall:
        x = x.transpose(1, 2)
    x = x / torch.sqrt(x.double().square().sum((1, 2), keepdim=True)).float()
    for _ in range(steps):
        g = torch.matmul(x, x.transpose(1, 2))
        x = a * x + torch.matmul(b * g + c * torch.matmul(g, g), x)
    return (x.transpose(1, 2) if tall else x).to(v.dtype)


def _plain(s):
    c = s["case"]
    if c["op"] == "embed":
        ids = s["ids"]
        rows = s["table"][ids.clamp(min=0)].float() * c["scale"]
        return torch.where((ids >= 0)[:, None], rows, torch.zeros((), device=ids.device)).to(DTYPES[c["dtype"]])
    if c["op"] == "embed_grad":
        ids = s["ids"]
        d = torch.zeros((c["V"] + 1, c["k"]), device=ids.device)
        d.index_add_(0, torch.where(ids >= 0, ids, c["V"]), s["dy"].float())
        return d[:-1] * c["scale"]
    if c["op"] == "norm":
        return _plain_norm(s, c)
    if c["op"] == "norm_grad":
        dy, h, r = s["dy"].float(), s["h"].float(), s["r"][:, None]
        g = dy * s["w"]
        dx = r * (g - h * (r * r * (g * h).mean(1, keepdim=True)))
        if s["dres"] is not None:
            dx = dx + s["dres"].float()
        return {"dx": dx.to(s["dy"].dtype), "dw": (dy * (h * r)).sum(0)}
    return _plain_orthogonal(s["v"], c["steps"])


# ---- the library's calls -------------------------------------------------------------------------

def _own(s):
    from paper_1901_08227_b200 import tng

    c = s["case"]
    if c["op"] == "embed":
        return tng.embed(s["table"], s["ids"], scale=c["scale"], dtype=DTYPES[c["dtype"]])
    if c["op"] == "embed_grad":
        return tng.embed_grad(s["dy"], s["ids"], c["V"], scale=c["scale"])
    if c["op"] == "norm":
        if c["codes"]:
            q, scale, h, r = tng.rmsnorm8(s["x"], s["w"], eps=EPS, residual=s["residual"])
            out = {"r": r, "q": q, "scale": scale}
        else:
            y, h, r = tng.rmsnorm(s["x"], s["w"], eps=EPS, residual=s["residual"])
            out = {"r": r, "y": y}
        if c["residual"]:
            out["h"] = h
        return out
    if c["op"] == "norm_grad":
        dx, dw = tng.rmsnorm_grad(s["dy"], s["h"], s["w"], s["r"], dres=s["dres"])
        return {"dx": dx, "dw": dw}
    return tng.orthogonalize(s["v"], steps=c["steps"], coefficients=COEFFICIENTS)


def run(state):
    return _own(state) if own else _plain(state)


def work(case):
    e = SIZE[case["dtype"]]
    if case["op"] == "embed":
        T, V, k = case["T"], case["V"], case["k"]
        return {"bytes": SIZE[case["table"]] * min(T, V) * k + 8 * T + e * T * k, "flops": T * k}
    if case["op"] == "embed_grad":
        T, V, k = case["T"], case["V"], case["k"]
        return {"bytes": e * T * k + 8 * T + 4 * V * k, "flops": T * k}
    if case["op"] == "norm":
        n = case["T"] * case["k"]
        return {"bytes": e * n * (3 if case["residual"] else 1) + (1 if case["codes"] else e) * n + 4 * case["k"] + 8 * case["T"], "flops": 6 * n}
    if case["op"] == "norm_grad":
        n = case["T"] * case["k"]
        return {"bytes": e * n * (4 if case["dres"] else 3) + 8 * case["k"] + 4 * case["T"], "flops": 10 * n}
    s, l = sorted((case["m"], case["n"]))
    # G and G^2 are symmetric: half of their entries are needed
    return {"bytes": 2 * e * case["batch"] * s * l, "flops": case["batch"] * case["steps"] * (3 * s * s * l + s ** 3)}


# ---- the definitions in 64 bits ------------------------------------------------------------------

def _exact_update(v, steps):
    """One matrix through its Gram matrix on the shorter side, all coefficients gathered in one polynomial of it."""
    a, b, c = COEFFICIENTS
    x = v.double()
    flip = x.shape[0] > x.shape[1]
    x = x.T.contiguous() if flip else x
    x = x / torch.linalg.vector_norm(x)
    eye = torch.eye(x.shape[0], dtype=torch.float64, device=x.device)
    for _ in range(steps):
        g = x @ x.T
        x = torch.addmm(a * x, (b * eye + c * g) @ g, x)
    return x.T if flip else x


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "embed":
        ids = s["ids"]
        y = torch.zeros((case["T"], case["k"]), dtype=torch.float64, device="cuda")
        live = torch.nonzero(ids >= 0)[:, 0]
        y[live] = s["table"][ids[live]].double() * case["scale"]
        return y
    if case["op"] == "embed_grad":
        ids, k = s["ids"], case["k"]
        out = torch.zeros((case["V"], k), dtype=torch.float64, device="cuda")
        live = torch.nonzero(ids >= 0)[:, 0]
        order = live[torch.argsort(ids[live], stable=True)]
        found, counts = torch.unique_consecutive(ids[order], return_counts=True)
        if found.numel() == 0:
            return out
        ends = torch.cumsum(counts, 0)
        for c0 in range(0, k, 512):              # sums of runs as differences of running sums
            run_sum = torch.cumsum(s["dy"][order, c0:c0 + 512].double(), 0)
            upto = run_sum[ends - 1]
            upto[1:] = upto[1:] - run_sum[ends - 1][:-1]
            out[found, c0:c0 + 512] = upto * case["scale"]
        return out
    if case["op"] == "norm":
        def single(v):                           # an fp32 operation that decides a code is part of the definition
            return v.to(torch.float32).to(torch.float64)

        h = s["x"].double()
        if case["residual"]:
            h = single(h + s["residual"].double()).to(s["x"].dtype).double()
        w = s["w"].double()
        r = torch.rsqrt((h * h).sum(1) / case["k"] + EPS)
        out = {"r": r}
        if case["residual"]:
            out["h"] = h
        if not case["codes"]:
            out["y"] = h * r[:, None] * w[None, :]
            return out
        t = single(h * w[None, :])
        top = t.abs().max(dim=1, keepdim=True).values
        out["q"] = single(t * single(127.0 / top)).round().to(torch.int8)
        out["scale"] = top[:, 0] / 127.0 * r
        return out
    if case["op"] == "norm_grad":
        dy, h, r, w = s["dy"].double(), s["h"].double(), s["r"].double()[:, None], s["w"].double()[None, :]
        z = h * r                                # the normed rows
        along = (dy * w * z).sum(1, keepdim=True) / case["k"]
        dx = (dy * w - z * along) * r
        if case["dres"]:
            dx = dx + s["dres"].double()
        return {"dx": dx, "dw": torch.einsum("tk,tk->k", dy, z)}
    return torch.stack([_exact_update(v, case["steps"]) for v in s["v"]])
