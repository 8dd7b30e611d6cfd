"""Pins of the restatement that the GPU tests of the training-layer operators compare with (CPU only)."""
import numpy as np
import pytest

import layers_ref as ref
import oracle


def test_uniforms_are_the_oracle_philox():
    seed, layer, step, row0 = 0x1234567890ABCDEF, 7, 99, 5
    u = ref.uniforms(3, 10, seed, layer, step, ref.TAG_ROUNDING, row0)
    for r in range(3):
        for c in range(10):
            w = oracle.philox4x32_10([c // 4, row0 + r, layer + ref.TAG_ROUNDING, step], [seed & 0xFFFFFFFF, seed >> 32])
            assert u[r, c] == oracle.uniform24(w[c % 4])


def test_codes_are_nearest_and_their_edges():
    rng = np.random.default_rng(0)
    x = rng.standard_normal((20, 300)).astype(np.float32)
    q, s = ref.codes(x)
    # |x - q s| <= s/2 up to the roundings of inv, the product and s (127 * 2^-22 of a step)
    assert np.all(np.abs(x - q.astype(np.float64) * s[:, None]) <= s[:, None] * (0.5 + 127 * 2.0 ** -22))
    assert np.array_equal(np.abs(q).max(1), np.full(20, 127))
    x[0] = 0; x[1, 3] = np.nan; x[2, 4] = -np.inf; x[3] *= np.float32(2.0 ** -125); x[3, 0] = 2.0 ** -121
    q, s = ref.codes(x)
    assert s[0] == 0 and not q[0].any() and np.isnan(s[1]) and not q[1].any() and np.isinf(s[2]) and not q[2].any()
    assert s[3] == 0 and not q[3].any()


def test_stochastic_codes_are_unbiased():
    # mean of n draws of a Bernoulli step: standard error at most s/(2 sqrt n); 6 of them over 64 values
    x = np.linspace(-1, 1, 64, dtype=np.float32)[None, :]
    n, total = 4000, np.zeros(64)
    for t in range(n):
        q, s = ref.codes(x, ref.uniforms(1, 64, 3, 1, t, ref.TAG_ROUNDING))
        total += q[0].astype(np.float64) * s[0]
    assert np.all(np.abs(total / n - x[0]) <= 6 * s[0] / (2 * np.sqrt(n)) + s[0] * 2.0 ** -16)


def test_linear_gradients_match_differences_up_to_the_coding_error():
    """f = sum(dy * (x W^T + b)) is linear in x, W and b: a difference quotient is its derivative exactly."""
    rng = np.random.default_rng(1)
    T, K, N = 9, 20, 13
    x, w = rng.standard_normal((T, K)).astype(np.float32), rng.standard_normal((N, K)).astype(np.float32)
    dy = rng.standard_normal((T, N)).astype(np.float32)
    wt, wts = ref.codes(w.T)
    dx, dw, db = ref.linear_grad(dy, x, wt, wts)

    def f(x, w, b):
        return float((dy.astype(np.float64) * (x @ w.T + b)).sum())

    x64, w64, b = x.astype(np.float64), w.astype(np.float64), np.zeros(N)
    sy, syc = np.abs(dy).max(1) / 127, np.abs(dy).max(0) / 127
    sx = np.abs(x).max(0) / 127
    h = 0.5
    for t, k in [(0, 0), (4, 7), (8, 19)]:
        e = np.zeros_like(x64); e[t, k] = h
        fd = (f(x64 + e, w64, b) - f(x64 - e, w64, b)) / (2 * h)
        # each factor is off by at most half a step: sum |dy| sw/2 + |w| sy/2 + sy sw/4
        bound = (np.abs(dy[t]) * wts[k] / 2 + np.abs(w[:, k]) * sy[t] / 2 + sy[t] * wts[k] / 4).sum() * 1.01
        assert abs(dx[t, k] - fd) <= bound
    for n, k in [(0, 0), (6, 11), (12, 19)]:
        e = np.zeros_like(w64); e[n, k] = h
        fd = (f(x64, w64 + e, b) - f(x64, w64 - e, b)) / (2 * h)
        bound = (np.abs(dy[:, n]) * sx[k] / 2 + np.abs(x[:, k]) * syc[n] / 2 + syc[n] * sx[k] / 4).sum() * 1.01
        assert abs(dw[n, k] - fd) <= bound
    for n in range(N):
        e = np.zeros(N); e[n] = h
        assert db[n] == pytest.approx((f(x64, w64, e) - f(x64, w64, -e)) / (2 * h), rel=1e-12, abs=1e-12)


def test_dropout_keeps_the_mean_and_its_gradient_is_the_difference():
    u = ref.uniforms(64, 1000, 11, 2, 3, ref.TAG_DROPOUT)
    for p in (0.0, 0.1, 0.5, 1.0):
        y = ref.dropout(np.ones((64, 1000)), p, u)
        kept = np.count_nonzero(y) / y.size
        assert abs(kept - (1 - p)) <= 6 * np.sqrt(p * (1 - p) / y.size)
    x, dy = np.random.default_rng(2).standard_normal((2, 64, 1000)).astype(np.float32)
    g = ref.dropout(dy, 0.5, u)
    e = np.zeros_like(x); e[5, 17] = 2.0; e[6, 18] = 2.0
    for at in ((5, 17), (6, 18)):
        d = np.zeros_like(x); d[at] = 2.0
        fd = (dy.astype(np.float64) * (ref.dropout(x + d, 0.5, u).astype(np.float64) - ref.dropout(x - d, 0.5, u))).sum() / 4
        assert g[at] == pytest.approx(fd, abs=1e-5)
