"""The float64 forms of the dense operators pinned to closed values and to differences; CPU only."""
import math

import numpy as np
import pytest

from oracle import dense_oracle as D


def _differences(f, x, h=1e-6):
    """d f / d x, f a scalar of the whole array."""
    g = np.zeros_like(x)
    for i in np.ndindex(*x.shape):
        a, b = x.copy(), x.copy()
        a[i] += h
        b[i] -= h
        g[i] = (f(a) - f(b)) / (2 * h)
    return g


@pytest.mark.parametrize("name", D.ACTS)
def test_activations_and_their_slopes(name):
    z = np.array([-30.0, -3.0, -1.0, -0.25, 0.3, 1.0, 2.5, 30.0])
    want = {"none": z, "relu": np.maximum(z, 0), "gelu": np.array([0.5 * v * math.erfc(-v / math.sqrt(2)) for v in z]),
            "gelu_tanh": z / (1 + np.exp(-2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3))), "silu": z / (1 + np.exp(-z))}[name]
    assert np.allclose(D.act(z, name), want, rtol=1e-9, atol=1e-12)
    assert np.allclose(D.act_slope(z, name), (D.act(z + 1e-6, name) - D.act(z - 1e-6, name)) / 2e-6, atol=1e-8)


@pytest.mark.parametrize("name", D.ACTS)
@pytest.mark.parametrize("first", [False, True])
def test_linear_gradients_against_differences(name, first):
    rng = np.random.default_rng(1)
    x, w, b, r = rng.standard_normal((3, 5)), rng.standard_normal((4, 5)), rng.standard_normal(4), rng.standard_normal((3, 4))
    c = rng.standard_normal((3, 4))
    y, z = D.linear(x, w, b, r, name, first)
    dz = c * D.act_slope(z, name)
    assert np.allclose(D.linear_grad_input(dz, w), _differences(lambda a: (c * D.linear(a, w, b, r, name, first)[0]).sum(), x), atol=1e-7)
    dw, db = D.linear_grad_weight(dz, x)
    assert np.allclose(dw, _differences(lambda a: (c * D.linear(x, a, b, r, name, first)[0]).sum(), w), atol=1e-7)
    assert np.allclose(db, _differences(lambda a: (c * D.linear(x, w, a, r, name, first)[0]).sum(), b), atol=1e-7)
    # with the layer before's activation in front of x
    u, add = rng.standard_normal((3, 5)), rng.standard_normal((3, 5))
    dx = D.linear_grad_input(c, w, u, name, add)
    assert np.allclose(dx - add, _differences(lambda a: (c * D.linear(D.act(a, name), w)[0]).sum(), u), atol=1e-7)


def test_layer_norm_gradients_against_differences():
    rng = np.random.default_rng(2)
    x, g, b, c = rng.standard_normal((3, 7)), rng.standard_normal(7), rng.standard_normal(7), rng.standard_normal((3, 7))
    dx, dg, db = D.layer_norm_grad(c, x, g)
    assert np.allclose(dx, _differences(lambda a: (c * D.layer_norm(a, g, b)[0]).sum(), x), atol=1e-7)
    assert np.allclose(dg, _differences(lambda a: (c * D.layer_norm(x, a, b)[0]).sum(), g), atol=1e-7)
    assert np.allclose(db, _differences(lambda a: (c * D.layer_norm(x, g, a)[0]).sum(), b), atol=1e-7)
    y, mean, rstd = D.layer_norm(np.array([[1.0, 3.0]]), eps=0.0)
    assert np.array_equal(y, [[-1.0, 1.0]]) and mean[0] == 2 and rstd[0] == 1


def test_distillation_against_differences_and_by_hand():
    rng = np.random.default_rng(3)
    s = rng.standard_normal((4, 9))
    idx = np.array([[2, 5, 8], [1, 1, 0], [3, -1, 9], [-1, -1, 12]])
    val = rng.standard_normal((4, 3))
    w = np.array([1.0, 0.5, 2.0, 1.0])
    for T in (1.0, 3.0):
        loss, grad = D.distill(s, idx, val, T, w)
        assert np.allclose(grad, _differences(lambda a: D.distill(a, idx, val, T, w)[0].sum(), s), atol=1e-7)
        assert loss[3] == 0 and not grad[3].any()
        assert np.allclose(grad.sum(1), 0, atol=1e-12)           # p and q both sum to one
        # one entry: p = 1, the loss is the cross entropy at that index
        lse = T * math.log(np.exp(s[2] / T).sum())
        assert loss[2] == pytest.approx(2.0 * T * (lse - s[2, 3]))
    # a teacher that stores everything and equals the network: no loss, no gradient
    loss, grad = D.distill(s, np.tile(np.arange(9), (4, 1)), s, 2.0)
    assert np.allclose(loss, 0, atol=1e-12) and np.allclose(grad, 0, atol=1e-12)
    assert not D.distill(s, idx, val, 1.0, np.zeros(4))[1].any()
