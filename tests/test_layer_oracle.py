"""Pins of the fp64 oracle of the layer norm, the expert-level balance and the 4-bit values (no GPU needed): gradients
against central differences, closed forms by hand."""
import numpy as np
import pytest

from oracle import layer_oracle as L
from oracle import smoes_oracle as O


def slope(f, x, v, h=1e-6):
    return (f(x + h * v) - f(x - h * v)) / (2 * h)


def test_norm_by_hand():
    Y, mean, rstd = L.norm(np.array([[1.0, 3.0], [5.0, 5.0]]), np.array([2.0, 1.0]), np.array([0.0, 10.0]), 0.25)
    assert np.allclose(mean, [2, 5]) and np.allclose(rstd, [1 / np.sqrt(1.25), 2])
    assert np.allclose(Y, [[-2 / np.sqrt(1.25), 10 + 1 / np.sqrt(1.25)], [0, 10]])


def test_norm_gradients():
    rng = np.random.default_rng(0)
    S, w, b, dY, r = rng.standard_normal((4, 7)), rng.standard_normal(7), rng.standard_normal(7), rng.standard_normal((4, 7)), rng.standard_normal((4, 7))
    _, mean, rstd = L.norm(S, w, b, 1e-3)
    dX, dw, db = L.norm_bwd(dY, S, mean, rstd, w, r)
    f = lambda S, w, b: (dY * L.norm(S, w, b, 1e-3)[0]).sum() + (r * S).sum()  # noqa: E731
    for _ in range(3):
        vS, vw, vb = rng.standard_normal(S.shape), rng.standard_normal(7), rng.standard_normal(7)
        assert np.isclose(slope(lambda x: f(x, w, b), S, vS), (dX * vS).sum(), rtol=1e-6)
        assert np.isclose(slope(lambda x: f(S, x, b), w, vw), (dw * vw).sum(), rtol=1e-6)
        assert np.isclose(slope(lambda x: f(S, w, x), b, vb), (db * vb).sum(), rtol=1e-6)


def test_balance_by_hand():
    """Two experts, one of them chosen by both tokens: f = (2, 0), P = mean g; a sample without selections adds nothing."""
    g = np.array([[0.75, 0.25], [0.5, 0.5], [0.1, 0.9]])
    loss, counts, d_gate, grad = L.expert_balance(g, np.array([[0], [0], [-1]]), [0, 2, 3], 3.0)
    assert counts.tolist() == [[2, 0], [0, 0]] and np.isclose(loss, (2 * 0.625) / 2)
    assert np.allclose(d_gate, [[3.0 * 2 / (2 * 2), 0], [0, 0]]) and np.allclose(grad, [[1.5, 0], [1.5, 0], [0, 0]])
    even = L.expert_balance(np.full((4, 4), 0.25), np.arange(4)[:, None], [0, 4])[0]
    assert np.isclose(even, 1.0)                        # everything even: 1, whatever E is


@pytest.mark.parametrize("gate", ["softmax", "sigmoid"])
def test_balance_gradient(gate):
    rng = np.random.default_rng(1)
    z, idx = rng.standard_normal((9, 5)), rng.integers(-1, 6, (9, 2))       # dropped ones and one that does not exist
    raw = lambda z: 1 / (1 + np.exp(-z))  # noqa: E731
    g = (lambda z: raw(z) / raw(z).sum(1, keepdims=True)) if gate == "sigmoid" else O.softmax_gate
    f = lambda z: 0.7 * L.expert_balance(g(z), idx, [0, 4, 9])[0]  # noqa: E731
    t = L.expert_balance(g(z), idx, [0, 4, 9], 0.7)[3]
    dz = L.gate_grad_logits(g(z), t, 1 - raw(z) if gate == "sigmoid" else 1.0)
    for _ in range(3):
        v = rng.standard_normal(z.shape)
        assert np.isclose(slope(f, z, v), (dz * v).sum(), rtol=1e-6)


def test_mx_values_stay_and_round_to_the_nearest():
    rng = np.random.default_rng(2)
    x = rng.standard_normal((6, 64)) * 2.0 ** rng.integers(-120, 120, (6, 1))
    q, s = L.mx_quantise(x)
    v = L.mx_values(q, s)
    again = L.mx_quantise(v)
    assert np.array_equal(L.mx_values(*again), v)
    scale = 2.0 ** (s.astype(float) - 127).repeat(32, 1)
    sizes = np.concatenate([L.MX_SIZES, -L.MX_SIZES])
    best = np.abs(x[..., None] - sizes * scale[..., None]).min(-1)
    assert np.allclose(np.abs(x - v), best, rtol=1e-12, atol=0)
