"""The fp64 oracle of the output layers against central differences of its own losses, and
the properties that pin it: a gradient's sum, a softmax's scale, padding rows."""
import math

import numpy as np
import pytest

from oracle import output_layers as ol


def differences(f, x, eps=1e-6):
    g = np.zeros_like(x)
    for i in np.ndindex(*x.shape):
        a, b = x.copy(), x.copy()
        a[i] += eps
        b[i] -= eps
        g[i] = (f(a) - f(b)) / (2 * eps)
    return g


def close(got, want):
    # central differences of a smooth fp64 function with step 1e-6: error about 1e-9 of its scale
    assert np.abs(got - want).max() <= 1e-7 * max(1.0, np.abs(want).max())


@pytest.mark.parametrize("R,N", [(1, 1), (3, 2), (4, 7)])
def test_norm_gradients(R, N):
    rng = np.random.default_rng(R * 10 + N)
    x, gamma, beta, dy = rng.normal(size=(R, N)), rng.normal(size=N), rng.normal(size=N), rng.normal(size=(R, N))
    loss = lambda x=x, g=gamma, b=beta: float((ol.norm_forward(x, g, b, 1e-3)[0] * dy).sum())
    _, m, r = ol.norm_forward(x, gamma, beta, 1e-3)
    dx, dg, db = ol.norm_backward(dy, x, gamma, m, r)
    close(dx, differences(lambda v: loss(x=v), x))
    close(dg, differences(lambda v: loss(g=v), gamma))
    close(db, differences(lambda v: loss(b=v), beta))


@pytest.mark.parametrize("name", ol.ACTS)
def test_linear_gradients(name):
    rng = np.random.default_rng(5)
    R, K, N = 3, 4, 5
    x, W, b, dy = rng.normal(size=(R, K)), rng.normal(size=(N, K)), rng.normal(size=N), rng.normal(size=(R, N))
    res, add = rng.normal(size=(R, N)), rng.normal(size=(R, K))
    loss = lambda x=x, W=W, b=b: float((ol.linear_forward(x, W, b, res, name)[0] * dy).sum())
    y, pre = ol.linear_forward(x, W, b, res, name)
    dx, dW, db, _ = ol.linear_backward(dy, x, W, pre, add, name)
    close(dx - add, differences(lambda v: loss(x=v), x))
    close(dW, differences(lambda v: loss(W=v), W))
    close(db, differences(lambda v: loss(b=v), b))


@pytest.mark.parametrize("tau,alpha", [(1.0, 1.0), (2.0, 0.5), (0.5, 0.75), (3.0, 0.0)])
def test_distill_gradient(tau, alpha):
    rng = np.random.default_rng(7)
    R, V, k = 4, 6, 3
    z, t = rng.normal(size=(R, V)), rng.normal(size=(R, k))
    idx = np.array([[0, 3, 5], [2, 2, 1], [-1, 4, -1], [-1, -1, -1]], np.int32)
    gold = np.array([1, 2, -1, -1], np.int32)
    loss, d = ol.distill(z, idx, t, gold, tau, alpha, 0.3)
    close(d, differences(lambda v: float(ol.distill(v, idx, t, gold, tau, alpha, 0.3)[0].sum()), z))
    assert np.abs(d.sum(1)).max() < 1e-14  # a softmax's gradient moves no mass
    assert loss[3] == 0 and not d[3].any()


def test_distill_of_an_agreeing_student_is_zero():
    z = np.log(np.array([[0.5, 0.25, 0.25]]))
    loss, d = ol.distill(z, np.array([[2, 0, 1]], np.int32), z[:, [2, 0, 1]], None, 1.0, 1.0, 1.0)
    assert abs(loss[0]) < 1e-15 and np.abs(d).max() < 1e-15


def test_distill_rows_without_logits_give_nothing():
    z = np.full((1, 3), -math.inf)
    loss, d = ol.distill(z, np.array([[0]], np.int32), np.zeros((1, 1)), np.array([1], np.int32), 1.0, 0.5, 1.0)
    assert loss[0] == 0 and not d.any()


def test_select_orders_ties_by_place():
    z = np.zeros((1, 2, 3), np.float32)
    s, p, t = ol.select(z, None, np.zeros((1, 2), np.float32), None)
    assert p.tolist() == [[0, 0]] and t.tolist() == [[0, 1]] and s.tolist() == [[0.0, 0.0]]
    s, p, t = ol.select(z, None, np.array([[-math.inf, -1.0]], np.float32), np.array([[0, 1]], np.uint8))
    assert p.tolist() == [[1, -1]] and t.tolist() == [[-1, -1]] and s[0, 1] == -math.inf


def test_push_and_reorder():
    rng = np.random.default_rng(1)
    S, B, K, H = 3, 1, 2, 2
    h, c = rng.normal(size=(S, 2, H)), rng.normal(size=(S, 2, H))
    p = np.array([1, 2], np.int32)
    po, ho, co, th, tc = ol.reorder(np.array([[1, 1]]), p, h, c, np.zeros_like(h), np.zeros_like(c))
    assert po.tolist() == [2, 2] and np.array_equal(ho[:, 0], h[:, 1]) and np.array_equal(th[0], h[2, 1])
    new = rng.normal(size=(2, H))
    p2, h2, _, top, _ = ol.push(np.array([1, -1], np.int8), new, new, p, h, c)
    assert p2.tolist() == [2, 1] and np.array_equal(h2[2, 0], new[0]) and np.array_equal(top[1], h[1, 1])
    p3, h3, _, _, _ = ol.push(np.array([0, 1], np.int8), new, new, p, h, c)  # row 1 is full
    assert p3.tolist() == [1, 2] and np.array_equal(h3, h)
