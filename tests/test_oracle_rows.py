"""Pins of the fp64 row operators: closed forms, invariances, and gradients
against central differences."""
import numpy as np
import pytest

from oracle import rows


def _diff(f, x, h):
    """Central differences of a scalar function of an array."""
    g = np.zeros_like(x)
    for i in np.ndindex(*x.shape):
        a, b = x.copy(), x.copy()
        a[i] += h
        b[i] -= h
        g[i] = (f(a) - f(b)) / (2 * h)
    return g


def test_layernorm_forward_closed_form():
    # the row 1, 3: mean 2, variance 1
    y, mean, rstd = rows.layernorm_forward([[1.0, 3.0]], [2.0, 4.0], [0.5, -0.5], 0.0)
    assert np.allclose(y, [[-1.5, 3.5]]) and mean[0] == 2.0 and rstd[0] == 1.0
    y, mean, rstd = rows.layernorm_forward([[5.0]], None, None, 0.25)      # one channel: nothing is left
    assert y[0, 0] == 0.0 and mean[0] == 5.0 and rstd[0] == 2.0


def test_layernorm_gradient_against_differences():
    rng = np.random.default_rng(1)
    x, gamma, beta, dy = rng.standard_normal((4, 7)), rng.standard_normal(7), rng.standard_normal(7), \
        rng.standard_normal((4, 7))
    _, mean, rstd = rows.layernorm_forward(x, gamma, beta, 1e-3)
    dx, dgamma, dbeta = rows.layernorm_backward(dy, x, gamma, mean, rstd)

    def f(x_, g_, b_):
        return (rows.layernorm_forward(x_, g_, b_, 1e-3)[0] * dy).sum()

    # central differences: truncation h^2 |f'''| / 6 and rounding 1e-16 |f| / h are both about 1e-9 at h = 1e-5
    assert np.allclose(dx, _diff(lambda v: f(v, gamma, beta), x, 1e-5), atol=1e-7)
    assert np.allclose(dgamma, _diff(lambda v: f(x, v, beta), gamma, 1e-5), atol=1e-7)
    assert np.allclose(dbeta, _diff(lambda v: f(x, gamma, v), beta, 1e-5), atol=1e-7)


def test_topk_orders_ties_zeros_and_nans():
    v, i = rows.topk([[1.0, 3.0, -0.0, 3.0, 0.0, np.nan, -np.inf]], 7)
    assert i.tolist() == [[5, 1, 3, 0, 2, 4, 6]]
    assert np.isnan(v[0, 0]) and v[0, 1] == 3.0 and v[0, 6] == -np.inf


def test_distill_is_zero_where_the_student_is_the_teacher():
    """All classes listed, the student's logits the teacher's own up to a
    shift, no labels: no loss and no gradient."""
    rng = np.random.default_rng(2)
    z = rng.standard_normal((3, 9)) * 3
    idx = np.tile(np.arange(9), (3, 1))
    row, loss, dz = rows.distill(z, z + 1.5, idx, None, None, 2.5, 1.0, 1.0)
    assert np.abs(row).max() < 1e-12 and np.abs(dz).max() < 1e-12 and abs(loss) < 1e-12


def test_distill_without_teacher_is_cross_entropy():
    z = np.log(np.array([[1.0, 2.0, 5.0]]))
    row, loss, dz = rows.distill(z, np.zeros((1, 0)), np.zeros((1, 0), int), [2], None, 4.0, 0.0, 0.5)
    assert np.isclose(row[0], -np.log(5 / 8)) and np.isclose(loss, 0.5 * row[0])
    assert np.allclose(dz, 0.5 * np.array([[1 / 8, 2 / 8, 5 / 8 - 1]]))


@pytest.mark.parametrize("alpha,temperature", [(1.0, 1.0), (0.3, 2.0), (0.7, 4.0)])
def test_distill_gradient_against_differences(alpha, temperature):
    """Short lists, a doubled class, an empty list, an absent label, a
    weight of zero."""
    rng = np.random.default_rng(3)
    z, t = rng.standard_normal((5, 8)) * 2, rng.standard_normal((5, 4)) * 2
    idx = np.array([[0, 3, 7, 2], [1, 1, 5, -1], [-1, -1, 8, -1], [4, 5, 6, 7], [2, 3, 4, 5]])
    t[3, 1] = -np.inf
    labels, weight = [3, -1, 2, 0, 1], [1.0, 0.5, 2.0, 1.5, 0.0]
    _, _, dz = rows.distill(z, t, idx, labels, weight, temperature, alpha, 0.2)
    num = _diff(lambda v: rows.distill(v, t, idx, labels, weight, temperature, alpha, 0.2)[1], z, 1e-5)
    assert np.allclose(dz, num, atol=1e-7)
    assert np.allclose(dz.sum(axis=1), 0.0, atol=1e-12)      # softmax gradients sum to zero
    assert not dz[4].any()


def test_distill_masked_classes_and_rows():
    z = np.array([[0.0, -np.inf, 1.0], [-np.inf] * 3])
    row, loss, dz = rows.distill(z, np.zeros((2, 1)), np.zeros((2, 1), int), None, None, 1.0, 1.0, 1.0)
    assert np.isclose(row[0], np.log(1 + np.e)) and row[1] == 0.0 and np.isclose(loss, row[0])
    assert dz[0, 1] == 0.0 and not dz[1].any()
