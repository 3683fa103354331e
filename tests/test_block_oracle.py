"""Pins of the float64 definitions of the norm, of the products by expert and of the row form in 8
bits in oracle/operators_oracle.py: closed forms, differences, and mistakes planted on the CPU that the
pins have to see."""
import numpy as np
import pytest

from oracle import operators_oracle as O


def test_norm_of_a_closed_form():
    y, r = O.rms_norm(np.array([[3.0, 4.0], [0.0, 0.0]]), np.array([1.0, 2.0]), 0.0 + 1e-300)
    assert np.allclose(r[0], 1 / np.sqrt(12.5)) and np.allclose(y[0], [3 / np.sqrt(12.5), 8 / np.sqrt(12.5)])
    assert np.all(y[1] == 0)
    h = np.random.default_rng(0).normal(0, 3, (4, 50))
    y, r = O.rms_norm(h, np.ones(50), 0.0)
    assert np.allclose((y * y).mean(1), 1)
    # a norm of the mean's removal instead is seen
    assert not np.allclose(((h - h.mean(1, keepdims=True)) * r[:, None]).var(1), 1, atol=1e-6)


@pytest.mark.parametrize("seed", range(3))
def test_norm_gradients_against_differences(seed):
    g = np.random.default_rng(seed)
    h, w, dy, dh = g.normal(0, 1, (3, 7)), g.normal(1, 0.3, 7), g.normal(0, 1, (3, 7)), g.normal(0, 1, (3, 7))
    eps = 0.01

    def loss(h, w):
        return np.sum(dy * O.rms_norm(h, w, eps)[0]) + np.sum(dh * h)

    dx, dw = O.rms_norm_backward(dy, h, O.rms_norm(h, w, eps)[1], w, dh)
    step = 1e-6
    for i in np.ndindex(*h.shape):
        e = np.zeros_like(h)
        e[i] = step
        assert abs((loss(h + e, w) - loss(h - e, w)) / (2 * step) - dx[i]) < 1e-7
    for i in range(7):
        e = np.zeros(7)
        e[i] = step
        assert abs((loss(h, w + e) - loss(h, w - e)) / (2 * step) - dw[i]) < 1e-7
    # the term of the row's own mean is not small
    assert np.abs(dx - dh - O.rms_norm(h, w, eps)[1][:, None] * dy * w).max() > 1e-2


@pytest.mark.parametrize("seed", range(3))
def test_products_and_their_gradients(seed):
    g = np.random.default_rng(seed)
    T, k, N, n_in, n_out = 5, 2, 3, 4, 6
    idx = np.sort(np.stack([g.choice(N, k, replace=False) for _ in range(T)]), 1)
    idx[1, 0] = -1
    offsets, row, route = O.dispatch_plan(idx, N)
    x, W = g.normal(0, 1, (T, n_in)), g.normal(0, 1, (N, n_out, n_in))
    out, mag = O.grouped_mm(x, W, offsets, route, k)
    for t in range(T):
        for s in range(k):
            if idx[t, s] >= 0:
                assert np.allclose(out[row[t, s]], W[idx[t, s]] @ x[t])
    assert np.all(out[offsets[N]:] == 0) and offsets[N] == T * k - 1
    assert np.all(mag >= np.abs(out) - 1e-12)
    # sorted rows give the same
    xs = O.dispatch(x, row)
    assert np.allclose(O.grouped_mm(xs, W, offsets)[0], out)
    # the gradients, against the bilinear form itself
    dy = g.normal(0, 1, out.shape)
    dx = O.grouped_mm_backward(dy, W, offsets)[0]
    dW = O.weight_grad(dy, x, offsets, route, k)[0]
    real = np.arange(T * k) < offsets[N]
    assert np.allclose((dx * xs)[real].sum(), (dy * out)[real].sum())
    assert np.allclose((dW * W).sum(), (dy * out)[real].sum())
    # another expert's weights are seen
    assert not np.allclose(O.grouped_mm(xs, np.roll(W, 1, 0), offsets)[0], out)


def test_step_of_the_row_form():
    s = O.row_scale(np.array([[127.0, -3.0], [0.0, 0.0], [np.inf, 1.0], [np.nan, 1.0]]))
    assert abs(s[0] - 1) <= 2.0 ** -23 and abs(s[1] * 127 * 2.0 ** 100 - 1) <= 2.0 ** -23
    assert np.isnan(s[2]) and np.isnan(s[3]) and np.all(s[:2] == s[:2].astype(np.float32))
