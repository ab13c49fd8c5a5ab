"""The definitions of oracle/worker.py against differences of their own forward direction, and against closed forms."""
import math

import numpy as np
import pytest

from oracle import worker as O


def differences(f, x, h=1e-5):
    """Central differences of the scalar f at x: error of h^2 / 6 times the third derivative, plus rounding of 1e-16 / h."""
    g = np.empty_like(x)
    flat, out = x.reshape(-1), g.reshape(-1)
    for i in range(flat.size):
        keep = flat[i]
        flat[i] = keep + h
        up = f()
        flat[i] = keep - h
        down = f()
        flat[i] = keep
        out[i] = (up - down) / (2 * h)
    return g


def close(a, b):
    assert np.abs(a - b).max() <= 1e-8 * max(1.0, np.abs(b).max()), np.abs(a - b).max()


def test_layer_norm_gradient_is_the_slope():
    rng = np.random.default_rng(0)
    x, w, b, r = rng.normal(0.5, 1.0, (3, 7)), rng.normal(1, 0.2, 7), rng.normal(0, 1, 7), rng.normal(0, 1, (3, 7))
    f = lambda: float((O.layer_norm(x, w, b, 1e-5)[0] * r).sum())  # noqa: E731
    _, mean, rstd = O.layer_norm(x, w, b, 1e-5)
    dx, dw, db = O.layer_norm_backward(r, x, w, mean, rstd)
    close(dx, differences(f, x))
    close(dw, differences(f, w))
    close(db, differences(f, b))


@pytest.mark.parametrize("kind", ["none", "relu", "gelu"])
def test_linear_gradients_are_the_slopes(kind):
    rng = np.random.default_rng(1)
    x, w, b, res = rng.normal(0, 1, (4, 5)), rng.normal(0, 1, (3, 5)), rng.normal(0, 1, 3), rng.normal(0, 1, (4, 3))
    r = rng.normal(0, 1, (4, 3))
    f = lambda: float((O.linear(x, w, b, kind, res)[0] * r).sum())  # noqa: E731
    z = O.linear(x, w, b)[1]
    dv = r * O.act_slope(z, kind)
    dw, db = O.linear_wgrad(dv, x)
    close(O.linear_dgrad(dv, w), differences(f, x))
    close(dw, differences(f, w))
    close(db, differences(f, b))
    close(r, differences(f, res))
    # through the activation in front of a layer: y = act(u) w^T
    u = rng.normal(0, 1, (4, 5))
    g = lambda: float((O.linear(O.act(u, kind), w)[0] * r).sum())  # noqa: E731
    close(O.linear_dgrad(r, w, kind, u), differences(g, u))


def test_distill_gradient_is_the_slope():
    rng = np.random.default_rng(2)
    s, t = rng.normal(0, 2, (4, 9)), rng.normal(0, 2, (4, 3))
    idx = np.array([[1, 5, 8], [0, -1, 3], [2, 2, 7], [-1, -1, -1]])
    dloss = np.array([1.0, 0.5, 2.0, 1.0])
    f = lambda: float((O.distill(s, idx, t, 2.0)[0] * dloss).sum()) * 0.25  # noqa: E731
    loss, grad = O.distill(s, idx, t, 2.0, dloss, 0.25)
    close(grad, differences(f, s))
    assert loss[3] == 0 and not grad[3].any()
    assert (loss[:2] > 0).all()   # a divergence of distinct indices


def test_distill_of_one_entry_is_the_cross_entropy():
    rng = np.random.default_rng(3)
    s = rng.normal(0, 1, (5, 11))
    label = np.array([[3], [0], [10], [5], [5]])
    loss, _ = O.distill(s, label, np.full((5, 1), 17.0), 1.0)
    want = [math.log(np.exp(r).sum()) - r[i[0]] for r, i in zip(s, label)]
    close(loss, np.array(want))


def test_distill_of_the_students_own_logits_is_zero():
    rng = np.random.default_rng(4)
    s = rng.normal(0, 1, (2, 6))
    loss, grad = O.distill(s, np.tile(np.arange(6), (2, 1)), s.copy(), 3.0)
    assert np.abs(loss).max() < 1e-14 and np.abs(grad).max() < 1e-14
