"""The references of the training step's tests against differences of the layer itself, in float64 (no GPU)."""
import numpy as np
import pytest

import train_ref as R


def layer(x, w, rt, k, gate, act):
    """sum_j gate FFN(x): [T, d]."""
    z, _ = R.first_product(x, w, rt, k, act)
    y = np.zeros_like(x)
    for e in range(len(rt["counts"])):
        sl = slice(rt["offsets"][e], rt["offsets"][e + 1])
        a = rt["perm"][sl]
        np.add.at(y, a // k, gate.reshape(-1)[a][:, None] * (R.hidden(z[sl], act) @ w["o"][e]))
    return y


@pytest.mark.parametrize("act", ["relu", "swiglu"])
def test_ffn_backward_against_differences(act):
    T, d, F, E, k = 9, 12, 8, 4, 2
    r = np.random.default_rng(5)
    x, dy, gate = r.standard_normal((T, d)), r.standard_normal((T, d)), r.random((T, k))
    w = {"a": r.standard_normal((E, d, F)), "o": r.standard_normal((E, F, d))}
    if act == "swiglu":
        w["b"] = r.standard_normal((E, d, F))
    rt = R.routing(T, k, E, 3, empty=(2,))
    z, _ = R.first_product(x, w, rt, k, act)
    (dxp, _), (dgate, _), dw = R.ffn_backward(x, dy, w, rt, k, gate, z, act)
    dx = np.zeros_like(x)
    np.add.at(dx, rt["perm"] // k, dxp)
    loss = lambda: (layer(x, w, rt, k, gate, act) * dy).sum()      # noqa: E731
    for value, grad in [(x, dx), (gate, dgate.reshape(T, k))] + [(w[n], dw[n][0]) for n in w]:
        for _ in range(4):
            v = r.standard_normal(value.shape)
            eps = 1e-6
            value += eps * v
            up = loss()
            value -= 2 * eps * v
            down = loss()
            value += eps * v
            assert abs((up - down) / (2 * eps) - (grad * v).sum()) < 1e-6 * np.abs(grad * v).sum()
    assert not dw["a"][0][2].any() and not dw["o"][0][2].any()


@pytest.mark.parametrize("renorm", [0, 1])
def test_route_backward_against_differences(renorm):
    r = np.random.default_rng(6)
    logits, c = r.standard_normal((5, 7)), r.standard_normal((5, 3))
    idx = np.argsort(-logits, axis=1)[:, :3]

    def gates(v):
        p = np.exp(v) / np.exp(v).sum(1, keepdims=True)
        g = np.take_along_axis(p, idx, 1)
        return g / g.sum(1, keepdims=True) if renorm else g

    dl = R.route_backward(logits, idx, gates(logits), c, renorm)
    for t in range(5):
        for e in range(7):
            v = np.zeros_like(logits)
            v[t, e] = 1e-6
            assert abs(((gates(logits + v) - gates(logits - v)) * c).sum() / 2e-6 - dl[t, e]) < 1e-8


def test_kept_values_bound():
    """The format by itself: 127 steps either side of zero, off by half a step."""
    v = np.random.default_rng(1).standard_normal((3, 130))
    m = R.block_max(v)
    q = np.rint(v * 127 / m)
    assert np.abs(q).max() == 127 and (np.abs(q * m / 127 - v) <= 0.5 * m / 127 * (1 + 1e-12)).all()
    assert R.restore(np.array([[127, -3]]), np.array([[0.5]])).tolist() == [[63.5, -1.5]]
