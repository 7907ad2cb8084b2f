"""The numpy oracle of the operators around the layers against values worked out by
hand and against differences."""
import numpy as np
import pytest

from oracle import training_oracle as O


def differences(f, x, step=1e-6):
    """df/dx of a scalar function, one entry at a time."""
    d = np.zeros(x.shape)
    for i in np.ndindex(x.shape):
        up, down = x.copy(), x.copy()
        up[i] += step
        down[i] -= step
        d[i] = (f(up) - f(down)) / (2 * step)
    return d


def test_norm_by_hand():
    y = O.norm([[1.0, 3.0, 5.0, 7.0]], eps=0.0)      # mean 4, variance 5
    assert np.allclose(y, np.array([[-3, -1, 1, 3]]) / np.sqrt(5), rtol=1e-15)
    y = O.norm([[1.0, 3.0]], weight=[2.0, 3.0], bias=[1.0, -1.0], eps=3.0, relu=True)     # r = 1/2
    assert y.tolist() == [[0.0, 0.5]]
    assert O.norm([[4.0]], bias=[0.25]).tolist() == [[0.25]]


@pytest.mark.parametrize("affine", [False, True])
def test_norm_gradient(affine):
    rng = np.random.default_rng(1)
    x, dz = rng.normal(size=(3, 7)), rng.normal(size=(3, 7))
    w, b = (rng.normal(size=7), rng.normal(size=7)) if affine else (None, None)
    dx, dw, db = O.norm_backward(dz, x, O.norm_stats(x, 1e-3), w)
    assert np.allclose(dx, differences(lambda v: (O.norm(v, w, b, 1e-3) * dz).sum(), x), atol=1e-7)
    if affine:
        assert np.allclose(dw, differences(lambda v: (O.norm(x, v, b, 1e-3) * dz).sum(), w), atol=1e-7)
        assert np.allclose(db, differences(lambda v: (O.norm(x, w, v, 1e-3) * dz).sum(), b), atol=1e-7)


def test_norm_gradient_behind_a_relu():
    rng = np.random.default_rng(2)
    u, dz = rng.normal(size=(4, 9)), rng.normal(size=(4, 9))
    x = np.maximum(u, 0)
    dx, _, _ = O.norm_backward(dz, x, O.norm_stats(x, 1e-3), zero=x == 0)
    assert np.allclose(dx, differences(lambda v: (O.norm(np.maximum(v, 0), eps=1e-3) * dz).sum(), u), atol=1e-7)


def test_lookup():
    table, ids = np.arange(12.0).reshape(4, 3), np.array([2, -1, 0, 2, 4])
    assert O.lookup(table, ids, 2.0).tolist() == [[12, 14, 16], [0, 0, 0], [0, 2, 4], [12, 14, 16], [0, 0, 0]]
    dy = np.random.default_rng(3).normal(size=(5, 3))
    assert np.allclose(O.lookup_grad(dy, ids, 4, 2.0), differences(lambda t: (O.lookup(t, ids, 2.0) * dy).sum(), table), atol=1e-7)


def test_distill_by_hand():
    # the teacher's one entry takes all: the loss is -log q of its class
    loss, dx = O.distill([[0.0, np.log(3.0)]], np.array([[1]]), [[5.0]])
    assert loss[0] == pytest.approx(-np.log(0.75)) and np.allclose(dx, [[0.25, -0.25]])
    # the same distribution on both sides
    loss, dx = O.distill([[1.0, 2.0, 4.0]], np.array([[2, 0, 1]]), [[4.0, 1.0, 2.0]], 2.0)
    assert loss[0] == pytest.approx(0.0, abs=1e-15) and np.allclose(dx, 0.0)
    # a class twice is two entries
    loss, dx = O.distill([[0.0, 0.0]], np.array([[0, 0]]), [[1.0, 1.0]])
    assert loss[0] == pytest.approx(np.log(0.5) - np.log(0.5)) and np.allclose(dx, [[-0.5, 0.5]])


def test_distill_rows_without_anything_to_learn():
    inf = np.inf
    x = np.array([[1.0, 2.0], [np.nan, 2.0], [-inf, -inf], [1.0, 2.0], [1.0, 2.0]])
    classes = np.array([[-1, 2], [0, 1], [0, 1], [0, 1], [0, -7]])
    t = np.array([[1.0, 1.0], [1.0, 1.0], [1.0, 1.0], [-inf, -inf], [0.0, np.nan]])
    loss, dx = O.distill(x, classes, t, 1.0, [1.0, 0.0, 1.0, 1.0, 1.0])
    assert (loss[:4] == 0).all() and (dx[:4] == 0).all()
    assert loss[4] > 0 and np.isfinite(dx).all()      # the entry outside may hold anything
    assert O.distill([[-inf, 1.0]], np.array([[0]]), [[1.0]])[0][0] == inf


def test_distill_gradient():
    rng = np.random.default_rng(4)
    x, t, w = rng.normal(size=(3, 6)), rng.normal(size=(3, 4)), np.array([1.0, 0.25, -2.0])
    classes = np.array([[0, 5, 2, -1], [3, 3, 1, 0], [6, -1, -1, 4]])
    _, dx = O.distill(x, classes, t, 1.7, w)
    assert np.allclose(dx, differences(lambda v: O.distill(v, classes, t, 1.7, w)[0].sum(), x), atol=1e-7)
