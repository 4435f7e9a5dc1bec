"""The oracle of the 8-bit layers with a scale for each token: worked numbers, properties, and its gradients against differences."""
import numpy as np
import pytest

from oracle import quant as Q
from oracle import t8 as O

F32 = np.float32


def test_codes_worked_example():
    q, s = O.codes([[127, -63.5, 0.5, 1.5, -0.5, -2.5], [0, 0, 0, 0, 0, 0], [254, 1, 3, 2, -1, -3]])
    assert np.array_equal(s, np.array([1, 1, 2], F32))
    assert np.array_equal(q, [[127, -64, 0, 2, 0, -2], [0] * 6, [127, 0, 2, 1, 0, -2]])


def test_codes_of_rows_that_are_not_finite():
    q, s = O.codes([[1, np.inf], [np.nan, 1], [1, -2]])
    assert np.isnan(s[:2]).all() and (q[:2] == 0).all() and s[2] == F32(2) / F32(127) and np.array_equal(q[2], [64, -127])


def test_codes_are_the_channel_wise_weight_quantiser():
    w = np.random.default_rng(0).standard_normal((33, 65)).astype(F32)
    q, s = O.codes(w)
    got = Q.weight_quant(w, 8)
    assert np.array_equal(got[0], q) and np.array_equal(got[1], s)


def test_codes_within_half_a_step():
    rng = np.random.default_rng(1)
    v = (rng.standard_normal((50, 300)) * np.exp(rng.uniform(-20, 20, (50, 1)))).astype(F32)
    q, s = O.codes(v)
    assert np.abs(q).max(1).min() == 127 and np.abs(q).max() == 127
    assert (np.abs(v - q * s.astype(np.float64)[:, None]) <= 0.5 * s[:, None] * (1 + 2.0 ** -16)).all()


def test_norm_has_unit_mean_square():
    h = np.random.default_rng(2).standard_normal((7, 1000)) * 3
    y = O.norm(h.astype(F32), None, 1e-12)
    assert np.allclose((y.astype(np.float64) ** 2).mean(1), 1, atol=1e-5)


@pytest.mark.parametrize("eps", [1e-6, 0.5])
def test_norm_gradient_against_differences(eps):
    """The scalar sum(g y) + sum(g2 h) of the float64 norm, central differences of 1e-5: errors of 1e-10 / 1e-5 and of (1e-5)^2."""
    rng = np.random.default_rng(3)
    h, w, g, g2 = rng.standard_normal((3, 11)), 1 + 0.3 * rng.standard_normal(11), rng.standard_normal((3, 11)), rng.standard_normal((3, 11))
    f = lambda h, w: float((g * h * O.rho(h, eps)[:, None] * w).sum() + (g2 * h).sum())  # noqa: E731
    dx, dw = O.norm_grad(h, w, eps, g, g2)
    d = 1e-5
    for i in range(3):
        for j in range(11):
            e = np.zeros_like(h)
            e[i, j] = d
            assert abs((f(h + e, w) - f(h - e, w)) / (2 * d) - dx[i, j]) < 1e-7
    for j in range(11):
        e = np.zeros_like(w)
        e[j] = d
        assert abs((f(h, w + e) - f(h, w - e)) / (2 * d) - dw[j]) < 1e-7


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_gates_and_their_gradient_against_differences(act):
    v = np.concatenate([np.linspace(-12, 12, 97), [-300.0, 300.0]])
    a, d = O.act(act, v)
    up, down = O.act(act, v + 1e-5)[0], O.act(act, v - 1e-5)[0]
    assert np.abs((up - down) / 2e-5 - d).max() < 1e-7
    plain = v / (1 + np.exp(-v)) if act == "silu" else 0.5 * v * (1 + np.tanh(np.sqrt(2 / np.pi) * (v + 0.044715 * v ** 3)))
    assert np.abs(a - plain).max() < 1e-12
    assert abs(a[-2]) <= 300 * np.exp(-300) and a[-1] == 300          # tanh gives 0 to both
    x, dv = np.random.default_rng(4).standard_normal((2, v.size))
    dx, dg = O.gated_grad(x, v, act, dv)
    assert np.array_equal(dx, dv * a) and np.allclose(dg, dv * x * d, rtol=1e-15)


def test_linear_and_its_gradient():
    rng = np.random.default_rng(5)
    qx, qw = rng.integers(-128, 128, (5, 32)), rng.integers(-128, 128, (7, 32))
    xs, ws, b = rng.uniform(0.1, 1, 5), rng.uniform(0.1, 1, 7), rng.standard_normal(7)
    X, W = qx * xs[:, None], qw * ws[:, None]
    assert np.allclose(O.linear(qx, xs, qw, ws, b), X @ W.T + b, rtol=1e-13)
    dy = rng.standard_normal((5, 7))
    assert np.allclose(O.linear_grad(dy, qw, ws), dy @ W, rtol=1e-13)
