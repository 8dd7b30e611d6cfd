"""Plain restatement of the training-layer operators in numpy: 64-bit sums, the fp32 operations that decide a
code written out one by one.  Shared by the CPU pins and the GPU tests."""
import numpy as np

TAG_ROUNDING, TAG_DROPOUT = 1 << 30, 1 << 31


def uniforms(rows, cols, seed, layer, step, tag, row0=0):
    """24-bit uniforms (float64) of a (rows, cols) array."""
    n4 = -(-cols // 4)
    m = np.uint64(0xFFFFFFFF)
    s32 = np.uint64(32)
    c = [np.broadcast_to(np.arange(n4, dtype=np.uint64), (rows, n4)),
         np.broadcast_to((np.arange(rows, dtype=np.uint64) + np.uint64(row0))[:, None], (rows, n4)),
         np.full((rows, n4), layer + tag, dtype=np.uint64), np.full((rows, n4), step, dtype=np.uint64)]
    k0, k1 = seed & 0xFFFFFFFF, seed >> 32
    for _ in range(10):
        p0, p1 = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(p1 >> s32) ^ c[1] ^ np.uint64(k0), p1 & m, (p0 >> s32) ^ c[3] ^ np.uint64(k1), p0 & m]
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    w = np.stack(c, axis=-1).reshape(rows, 4 * n4)[:, :cols]
    return (w >> np.uint64(8)).astype(np.float64) * 2.0 ** -24


def codes(x, u=None):
    """Lines are the rows of x (float32 values): int8 codes and float32 scales."""
    x = np.asarray(x, dtype=np.float32)
    with np.errstate(all="ignore"):
        top = np.max(np.abs(x), axis=1).astype(np.float32)          # NaN wins
        scale = (top / np.float32(127)).astype(np.float32)
        inv = (np.float32(127) / top).astype(np.float32)
        v = (x * inv[:, None]).astype(np.float32)
        q = np.rint(v) if u is None else np.clip(np.floor((v + u.astype(np.float32)).astype(np.float32)), -127, 127)
    zero = top < np.float32(2.0 ** -120)
    dead = zero | ~np.isfinite(top)
    scale[zero] = 0
    q[dead] = 0
    return q.astype(np.int8), scale


def product(a, sa, b, sb, bias=None):
    """The product before its last rounding, in float32 steps from the exact integer sum."""
    with np.errstate(all="ignore"):
        acc = a.astype(np.int64) @ b.astype(np.int64).T if a.size * b.shape[0] < 1 << 24 else \
            np.rint(a.astype(np.float64) @ b.astype(np.float64).T)
        y = acc.astype(np.float32) * sa[:, None].astype(np.float32)
        y = (y * sb[None, :].astype(np.float32)).astype(np.float32)
        return y if bias is None else (y + bias[None, :].astype(np.float32)).astype(np.float32)


def linear(x, wq, ws, bias=None):
    q, s = codes(x)
    return product(q, s, wq, ws, bias)


def linear_grad(dy, x, wt, wts, u=None):
    """(dx, dw, db): float32 steps, db in float64."""
    q, s = codes(dy, u)
    dx = product(q, s, wt, wts)
    qy, sy = codes(np.ascontiguousarray(dy.T), None if u is None else np.ascontiguousarray(u.T))
    qx, sx = codes(np.ascontiguousarray(x.T))
    return dx, product(qy, sy, qx, sx), np.asarray(dy, dtype=np.float64).sum(axis=0)


def dropout(x, p, u, residual=None):
    """Before the last rounding, float32 steps."""
    p = np.float32(p)
    x = np.asarray(x, dtype=np.float32)
    keep = np.float32(0) if p == 1 else np.float32(1) / (np.float32(1) - p)
    with np.errstate(all="ignore"):
        y = np.where(u >= np.float64(p), (x * keep).astype(np.float32), np.float32(0))
        return y if residual is None else (np.asarray(residual, dtype=np.float32) + y).astype(np.float32)
