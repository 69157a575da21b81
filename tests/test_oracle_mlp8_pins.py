"""Pins of the oracle of the MLP operators: known values, derivatives against differences, experts against one written out."""
import math

import numpy as np
import pytest

from oracle import mlp8

X = np.concatenate([np.linspace(-9, 9, 181) + 0.013, [0.25, -0.25, 1e-3, -1e-3, 30.0, -30.0]])


@pytest.mark.parametrize("act", mlp8.ACTS)
def test_slope_is_the_values_difference(act):
    h = 1e-6
    d = (mlp8.value(act, X + h) - mlp8.value(act, X - h)) / (2 * h)
    assert np.abs(d - mlp8.slope(act, X)).max() < 1e-7


def test_known_values():
    for x in (-3.0, -0.5, 0.0, 1.0, 2.5):
        a = np.array([x])
        assert mlp8.value("gelu", a)[0] == pytest.approx(0.5 * x * (1 + math.erf(x / math.sqrt(2))), abs=1e-15)
        t = math.tanh(math.sqrt(2 / math.pi) * (x + 0.044715 * x ** 3))
        assert mlp8.value("gelu_tanh", a)[0] == pytest.approx(0.5 * x * (1 + t), abs=1e-15)
        assert mlp8.value("silu", a)[0] == pytest.approx(x / (1 + math.exp(-x)), abs=1e-15)
        assert mlp8.value("relu", a)[0] == max(x, 0)
    assert mlp8.value("none", X) is not X and np.array_equal(mlp8.value("none", X), X)


@pytest.mark.parametrize("act", mlp8.ACTS)
def test_backward_is_the_forwards_difference(act):
    rng = np.random.default_rng(1)
    z, mul, dh = rng.standard_normal((3, 5, 7))
    du, dmul, db = mlp8.backward(dh, z, act, mul)
    h = 1e-6
    loss = lambda z_, m_: (dh * mlp8.forward(z_, act, m_, 2.0)).sum()
    for i, j in ((0, 0), (4, 6), (2, 3)):
        e = np.zeros((5, 7))
        e[i, j] = h
        assert (loss(z + e, mul) - loss(z - e, mul)) / (2 * h) == pytest.approx(du[i, j], abs=1e-8)
        assert (loss(z, mul + e) - loss(z, mul - e)) / (2 * h) == pytest.approx(dmul[i, j], abs=1e-8)
    e = np.zeros(7)
    e[2] = h
    assert (loss(z + e, mul) - loss(z - e, mul)) / (2 * h) == pytest.approx(db[2], abs=1e-8)


def test_route_takes_the_lower_expert_first():
    x, w = np.array([[1.0, 0.0], [0.0, 2.0]]), np.array([[1.0, 0.0], [3.0, 1.0], [3.0, 1.0], [0.0, 1.0]])
    ids, p = mlp8.route(x, w, 2, False)
    assert ids.tolist() == [[1, 2], [1, 2]]
    e = np.exp([1.0, 3.0, 3.0, 0.0])
    assert p[0] == pytest.approx([e[1] / e.sum()] * 2)
    assert mlp8.route(x, w, 2, True)[1] == pytest.approx(np.full((2, 2), 0.5))


def test_experts_written_out():
    gate, up, down = [np.array([[1.0, 2.0]])], [np.array([[3.0, -1.0]])], [np.array([[2.0], [5.0]])]
    x = np.array([[1.0, 1.0]])
    h = 3 / (1 + math.exp(-3)) * 2
    y = mlp8.experts(x, gate, up, down, [[0, 0, 1, -1]], [[0.5, 0.25, 9.0, 9.0]], "silu")
    assert y[0] == pytest.approx([0.75 * 2 * h, 0.75 * 5 * h])
