"""Pins of the float64 definitions in oracle/operators_oracle.py, which the GPU tests
compare with: closed forms, brute force, central differences, and planted mistakes that
the pins have to see (planted in the oracle's inputs and outputs, on the CPU)."""
import numpy as np
import pytest

from oracle import operators_oracle as O


def policy_inputs(seed, T=7, V=11):
    g = np.random.default_rng(seed)
    z = g.normal(0, 2, (T, V))
    y = g.integers(0, V, T)
    logp = O.token_stats(z, y, 0.8)[0]
    return dict(logits=z, token=y, logp_old=logp - g.normal(0, 0.5, T), adv=g.normal(0, 1, T),
                logp_ref=logp + g.normal(0, 0.3, T), weight=g.uniform(0.1, 1, T), kl_coef=0.3,
                inv_temp=0.8)


def test_log_probabilities_of_a_closed_form():
    z = np.log(np.array([[1.0, 2.0, 5.0], [4.0, 4.0, 0.0001]]))
    logp, lse, ent, p = O.token_stats(z, [2, 0])
    assert np.allclose(logp, [np.log(5 / 8), np.log(4 / 8.0001)])
    assert np.allclose(lse, np.log([8, 8.0001]))
    assert np.allclose(p.sum(1), 1)
    assert np.allclose(ent[0], -(1 / 8 * np.log(1 / 8) + 2 / 8 * np.log(2 / 8) + 5 / 8 * np.log(5 / 8)))
    # an id of probability 0 changes nothing, and rows without a distribution have none
    z2 = np.concatenate([z, np.full((2, 1), -np.inf)], 1)
    assert np.allclose(O.token_stats(z2, [2, 0])[0], logp)
    empty = O.token_stats(np.full((1, 3), -np.inf), [1])
    assert empty[0][0] == 0 and empty[1][0] == -np.inf and np.all(empty[3] == 0)


@pytest.mark.parametrize("seed", range(4))
def test_policy_gradient_against_differences(seed):
    kw = policy_inputs(seed)
    out = O.policy_loss(**kw)
    z = kw["logits"]
    num = np.zeros_like(z)
    h = 1e-6
    for t in range(z.shape[0]):
        for v in range(z.shape[1]):
            for sign in (1, -1):
                z2 = z.copy()
                z2[t, v] += sign * h
                num[t, v] += sign * O.policy_loss(**{**kw, "logits": z2})["sums"][0] / (2 * h)
    assert np.abs(num - out["dlogits"]).max() < 1e-8
    # the same with a wrong coefficient is seen
    assert np.abs(num - 1.01 * out["dlogits"]).max() > 1e-5


def test_policy_loss_on_policy_is_the_policy_gradient():
    kw = policy_inputs(9)
    kw.update(logp_old=O.token_stats(kw["logits"], kw["token"], 0.8)[0], logp_ref=None)
    out = O.policy_loss(**kw)
    assert np.isclose(out["sums"][0], -np.sum(kw["weight"] * kw["adv"]))
    assert np.allclose(out["coef"], -kw["weight"] * kw["adv"])
    assert out["sums"][2] == 0 and np.allclose(out["dlogits"].sum(1), 0)


def test_clipping_by_sign_of_the_advantage():
    z, y = np.zeros((1, 2)), np.array([0])
    for A, moved, stops in ((1, 0.5, True), (1, -0.5, False), (-1, -0.5, True), (-1, 0.5, False)):
        out = O.policy_loss(z, y, np.array([np.log(0.5) - moved]), np.array([A]))
        assert (out["coef"][0] == 0) == stops and out["sums"][2] == float(stops)


def test_plan_sorts_stably_and_inverts():
    g = np.random.default_rng(3)
    idx = g.integers(-1, 6, (50, 4))
    off, row, route = O.dispatch_plan(idx, 5)
    flat = idx.reshape(-1)
    kept = np.nonzero((flat >= 0) & (flat < 5))[0]
    assert off[-1] == len(kept)
    assert np.array_equal(route[:off[-1]], kept[np.argsort(flat[kept], kind="stable")])
    assert np.all(route[off[-1]:] == -1)
    for q in kept:
        assert route[row.reshape(-1)[q]] == q


def test_gradients_of_the_rows_are_the_transposes():
    g = np.random.default_rng(5)
    T, k, d, N = 9, 3, 4, 4
    _, row, _ = O.dispatch_plan(g.integers(-1, N, (T, k)), N)
    x, dxs = g.normal(size=(T, d)), g.normal(size=(T * k, d))
    # <dispatch(x), dxs> = <x, dispatch_backward(dxs)>
    assert np.isclose(np.sum(O.dispatch(x, row) * dxs), np.sum(x * O.combine(dxs, row)))
    o, gate, dy = g.normal(size=(T * k, d)), g.normal(size=(T, k)), g.normal(size=(T, d))
    d_o, dgate = O.combine_backward(dy, o, row, gate)
    h = 1e-6
    for name, arr, grad in (("o", o, d_o), ("gate", gate, dgate)):
        v = g.normal(size=arr.shape)
        up, down = arr + h * v, arr - h * v
        f = [np.sum(dy * O.combine(a if name == "o" else o, row, a if name == "gate" else gate))
             for a in (up, down)]
        assert np.isclose((f[0] - f[1]) / (2 * h), np.sum(grad * v), atol=1e-6)


def test_packed_form():
    g = np.random.default_rng(6)
    x = (g.normal(size=(40, 70)) * np.exp(g.normal(0, 6, (40, 1)))).astype(np.float32)
    q, s = O.pack(x)
    v = O.unpack(q, s)
    assert np.abs(q).max() <= 127 and s.min() >= 1
    step = np.repeat(np.exp2(s - 127.0), 32, axis=1)[:, :70]
    top = np.repeat(np.stack([np.abs(x[:, c:c + 32]).max(1) for c in (0, 32, 64)], 1), 32, 1)[:, :70]
    assert np.all(step <= top / 64) and np.all(step > top / 128.0001)
    # half a step, a whole one where a magnitude above 127.5 steps was cut to 127
    assert np.all(np.abs(v - x) <= np.where(np.abs(x) > 127.5 * step, 1.0, 0.5) * step)
    # packing the values again changes nothing
    q2, s2 = O.pack(v)
    assert np.array_equal(O.unpack(q2, s2), v)
    bad = x.copy()
    bad[3, 40] = np.nan
    bad[4, 1] = -np.inf
    v2 = O.unpack(*O.pack(bad))
    assert np.isnan(v2[3, 32:64]).all() and np.isnan(v2[4, :32]).all()
    assert np.array_equal(np.isnan(v2).sum(), 64)
    zero = O.pack(np.zeros((1, 5)))
    assert np.all(zero[0] == 0) and np.all(zero[1] == 1)


def test_swiglu_backward_against_differences():
    g = np.random.default_rng(7)
    a, u, dh = g.normal(0, 3, 50), g.normal(size=50), g.normal(size=50)
    da, du, h = O.swiglu_backward(a, u, dh)
    e = 1e-6
    assert np.allclose(h, O.swiglu(a, u))
    assert np.allclose(da, dh * (O.swiglu(a + e, u) - O.swiglu(a - e, u)) / (2 * e), atol=1e-8)
    assert np.allclose(du, dh * (O.swiglu(a, u + e) - O.swiglu(a, u - e)) / (2 * e), atol=1e-8)


def test_weight_grad_against_differences():
    g = np.random.default_rng(8)
    T, k, N, n_out, n_in = 6, 2, 3, 4, 5
    off, _, route = O.dispatch_plan(g.integers(-1, N, (T, k)), N)
    x, dy = g.normal(size=(T, n_in)), g.normal(size=(T * k, n_out))
    dW, mag = O.weight_grad(dy, x, off, route, k)
    W, v = g.normal(size=dW.shape), g.normal(size=dW.shape)

    def loss(W):        # <dy, x W^T> over the rows of every expert
        return sum(dy[r] @ (W[e] @ x[route[r] // k]) for e in range(N) for r in range(off[e], off[e + 1]))

    h = 1e-4
    assert np.isclose((loss(W + h * v) - loss(W - h * v)) / (2 * h), np.sum(dW * v))
    assert np.all(np.abs(dW) <= mag + 1e-12)
