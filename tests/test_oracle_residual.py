"""Pins of the fp64 oracle of the residual-block operators: RMS norm and linear
attention against closed forms, the quadratic form, and differences."""
import numpy as np
import pytest

from oracle import linattn, philox, rows


def test_rmsnorm_closed_form():
    h = np.array([[3.0, -4.0], [0.0, 0.0]])
    y, rstd = rows.rmsnorm_forward(h, np.array([2.0, 0.5]), 0.0 + 1e-300)
    assert np.allclose(y[0], [3 / np.sqrt(12.5) * 2, -4 / np.sqrt(12.5) * 0.5]) and np.all(y[1] == 0)
    assert np.isclose(rstd[0], 1 / np.sqrt(12.5))


def test_rmsnorm_backward_against_differences():
    rng = np.random.default_rng(0)
    h, dy, gamma = rng.standard_normal((3, 7)), rng.standard_normal((3, 7)), rng.standard_normal(7)
    f = lambda h, g: (rows.rmsnorm_forward(h, g, 1e-5)[0] * dy).sum()
    dh, dgamma = rows.rmsnorm_backward(dy, None, h, gamma, rows.rmsnorm_forward(h, gamma, 1e-5)[1])
    for _ in range(5):
        a, b, e = rng.standard_normal(h.shape), rng.standard_normal(7), 1e-6
        num = (f(h + e * a, gamma + e * b) - f(h - e * a, gamma - e * b)) / (2 * e)
        assert np.isclose(num, (dh * a).sum() + (dgamma * b).sum(), rtol=1e-7, atol=1e-7)


def test_dropout_factor_is_the_classifiers_mask_for_widths_of_four():
    keep = philox.dropout_keep(77, 3, 9, 12, 0.3)
    assert np.array_equal(rows.dropout_factor(77, 3, 9, 12, 0.3) != 0, keep)
    odd = rows.dropout_factor(77, 3, 9, 10, 0.3)
    assert np.array_equal(odd != 0, keep[:, :10])     # (counters by row: 10 columns take 12 words)
    big = rows.dropout_factor(1, 0, 400, 1000, 0.25)
    assert abs((big == 0).mean() - 0.25) < 4 * np.sqrt(0.25 * 0.75 / 4e5)


def _quadratic(q, k, v, g, s0, scale):
    T = q.shape[1]
    i = np.arange(T)
    lag = i[:, None] - i[None, :]
    w = np.where(lag >= 0, np.exp(g[:, None, None] * np.maximum(lag, 0)), 0.0)
    p = np.einsum("bihm,bjhm->bhij", q, k) * w
    o = np.einsum("bhij,bjhn->bihn", p, v)
    return scale * (o + np.einsum("bihm,bhmn,hi->bihn", q, s0, np.exp(g[:, None] * (i + 1))))


def test_linear_attention_is_its_quadratic_form():
    rng = np.random.default_rng(1)
    q, k, v = (rng.standard_normal((2, 9, 3, d)) for d in (4, 4, 5))
    s0, g = rng.standard_normal((2, 3, 4, 5)), np.log([0.9, 0.5, 1.0])
    o, sT, _ = linattn.forward(q, k, v, g, None, s0, 0.7)
    assert np.allclose(o, _quadratic(q, k, v, g, s0, 0.7))
    # in two pieces, the second from the first one's state
    a, s, _ = linattn.forward(q[:, :4], k[:, :4], v[:, :4], g, None, s0, 0.7)
    b, s, _ = linattn.forward(q[:, 4:], k[:, 4:], v[:, 4:], g, None, s, 0.7)
    assert np.allclose(np.concatenate([a, b], axis=1), o) and np.allclose(s, sT)


@pytest.mark.parametrize("lengths", [None, [5, 0], [1, 3]])
def test_linear_attention_backward_against_differences(lengths):
    rng = np.random.default_rng(2)
    B, T, H, Hk, Dk, Dv = 2, 5, 4, 2, 3, 2
    x = [rng.standard_normal(s) for s in ((B, T, H, Dk), (B, T, Hk, Dk), (B, T, Hk, Dv), (B, H, Dk, Dv))]
    do, dsT, g = rng.standard_normal((B, T, H, Dv)), rng.standard_normal((B, H, Dk, Dv)), np.log([0.9, 0.3, 1.0, 0.7])

    def f(q, k, v, s0):
        o, sT, _ = linattn.forward(q, k, v, g, lengths, s0, 0.6)
        return (o * do).sum() + (sT * dsT).sum()

    grads = linattn.backward(*x[:3], do, g, lengths, x[3], dsT, 0.6)
    for _ in range(4):
        d, e = [rng.standard_normal(a.shape) for a in x], 1e-6
        num = (f(*[a + e * b for a, b in zip(x, d)]) - f(*[a - e * b for a, b in zip(x, d)])) / (2 * e)
        assert np.isclose(num, sum((a * b).sum() for a, b in zip(grads, d)), rtol=1e-7, atol=1e-7)
