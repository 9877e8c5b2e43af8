"""The float64 oracle of the head's loss and the block norm against small sums
written out and against differences."""

import math

import numpy as np
import pytest

from oracle import head as O


def test_cross_entropy_by_hand():
    h, w = np.array([[1.0, 2.0]]), np.array([[0.5, 0.0], [0.0, 0.25], [1.0, -1.0]])
    z = [0.5, 0.5, -1.0]
    total = sum(math.exp(v) for v in z)
    for y in range(3):
        assert O.loss(h, w, np.array([y]))[0] == pytest.approx(math.log(total) - z[y], rel=1e-14)
    for y in (-100, 3):
        assert O.loss(h, w, np.array([y]))[0] == 0.0


def test_distillation_by_hand():
    h, w = np.array([[1.0, 2.0]]), np.array([[0.5, 0.0], [0.0, 0.25], [1.0, -1.0]])
    tau, alpha = 2.0, 0.25
    s = [math.exp(v / tau) for v in (0.5, 0.5, -1.0)]
    s = [v / sum(s) for v in s]
    q = [math.exp(v / tau) for v in (3.0, 1.0)]
    q = [v / sum(q) for v in q]
    kl = q[0] * math.log(q[0] / s[2]) + q[1] * math.log(q[1] / s[0])
    ids, top = np.array([[2, -1, 0, 1]]), np.array([[3.0, 9.0, 1.0, -math.inf]])
    got = O.loss(h, w, np.array([1]), ids, top, alpha, tau)[0]
    ce = O.loss(h, w, np.array([1]))[0]
    assert got == pytest.approx((1 - alpha) * ce + alpha * tau ** 2 * kl, rel=1e-13)
    assert O.loss(h, w, np.array([7]), ids, np.full((1, 4), -math.inf))[0] == 0.0


@pytest.mark.parametrize("tau,alpha", [(1.0, 0.5), (3.0, 0.2), (0.5, 1.0)])
@pytest.mark.parametrize("teacher", [False, True])
def test_gradients_against_differences(teacher, tau, alpha):
    g = np.random.default_rng(1)
    h, w = g.normal(size=(5, 3)), g.normal(size=(7, 3))
    y, dl = np.array([0, 6, -1, 3, 9]), g.normal(size=5)
    t = {}
    if teacher:
        ids = g.integers(0, 7, (5, 4))
        ids[1] = 7
        ids[2, 1:] = ids[2, 0]
        ids[4] = -1
        t = dict(ids=ids, top=g.normal(size=(5, 4)), alpha=alpha, tau=tau)
    dh, dw = O.loss_bwd(h, w, y, dl, **t)
    total = lambda h, w: float(O.loss(h, w, y, **t) @ dl)  # noqa: E731
    for a, d, f in ((h, dh, lambda x: total(x, w)), (w, dw, lambda x: total(h, x))):
        for i in np.ndindex(a.shape):
            e = np.zeros_like(a)
            e[i] = 1e-5
            assert (f(a + e) - f(a - e)) / 2e-5 == pytest.approx(d[i], rel=1e-7, abs=1e-8)


def test_norm_gradients_against_differences():
    g = np.random.default_rng(2)
    r, y, w = g.normal(size=(3, 4)), g.normal(size=(3, 4)), g.normal(size=4)
    dx, ds = g.normal(size=(3, 4)), g.normal(size=(3, 4))

    def total(r, w):
        x, s = O.norm(r, y, w, 1e-3)
        return float((x * dx).sum() + (s * ds).sum())

    dr, dw = O.norm_bwd(r + y, w, dx, ds, 1e-3)
    for a, d, f in ((r, dr, lambda x: total(x, w)), (w, dw, lambda x: total(r, x))):
        for i in np.ndindex(a.shape):
            e = np.zeros_like(a)
            e[i] = 1e-5
            assert (f(a + e) - f(a - e)) / 2e-5 == pytest.approx(d[i], rel=1e-7, abs=1e-8)


def test_teacher_of_the_lowest_values():
    """A number added to all of a token's logits changes nothing, whatever its size."""
    ids = np.array([[1, 2, 3, 4], [1, 2, 3, -1]])
    for dtype in (np.float32, np.float16):
        lo = float(np.finfo(dtype).min)
        for tau in (0.5, 2.0 ** -10, 2.0):
            q, some = O.teacher(5, ids, np.full((2, 4), lo), tau)
            assert some.all()
            assert np.allclose(q, [[0.25] * 4, [1 / 3, 1 / 3, 1 / 3, 0.0]], rtol=1e-15)
            q, _ = O.teacher(5, ids, np.array([[2.0, lo, lo, lo], [2.0, 2.0, lo, 2.0]]), 0.5)
            assert np.allclose(q, [[1, 0, 0, 0], [0.5, 0.5, 0, 0]], rtol=1e-15)
