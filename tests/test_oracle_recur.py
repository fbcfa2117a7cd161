"""Pins of the recurrence's 64-bit oracle: differences against its gradient, and hand-made cases."""

import numpy as np
import pytest

from oracle import recur


def _case(T, B, D, seed, done=False, lens=False):
    g = np.random.default_rng(seed)
    c = dict(x=g.normal(size=(T, B, D)), r=g.normal(size=(T, B, D)), i=g.normal(size=(T, B, D)),
             lam=g.uniform(-6, 1, D), h0=g.normal(size=(B, D)))
    c["done"] = (g.random((T, B)) < 0.2).astype(np.uint8) if done else None
    c["lens"] = g.integers(0, T + 1, B).astype(np.int32) if lens else None
    return c


def test_one_step_by_hand():
    one = np.ones((1, 1, 1))
    lam = np.zeros(1)
    y, h = recur.forward(2 * one, 0 * one, 0 * one, lam, h0=np.full((1, 1), 3.0))
    a = 2.0 ** -4                       # exp(-8 ln 2 / 2)
    assert y[0, 0, 0] == pytest.approx(a * 3.0 + np.sqrt(1 - a * a) * 1.0, rel=1e-14)
    assert h[0, 0] == y[0, 0, 0]


def test_an_episodes_end_starts_again_from_zero():
    c = _case(9, 1, 3, 1)
    done = np.zeros((9, 1), np.uint8)
    done[3] = 1
    y, h = recur.forward(c["x"], c["r"], c["i"], c["lam"], c["h0"], done)
    tail, _ = recur.forward(c["x"][4:], c["r"][4:], c["i"][4:], c["lam"])
    assert np.array_equal(y[4:], tail) and np.array_equal(h, tail[-1])
    done[8] = 1
    assert not recur.forward(c["x"], c["r"], c["i"], c["lam"], c["h0"], done)[1].any()


def test_lengths_end_a_sequence():
    c = _case(7, 3, 2, 2)
    lens = np.array([0, 4, 7], np.int32)
    y, h = recur.forward(c["x"], c["r"], c["i"], c["lam"], c["h0"], None, lens)
    assert not y[:, 0].any() and np.array_equal(h[0], c["h0"][0])
    part, last = recur.forward(*(c[k][:4, 1:2] for k in "xri"), c["lam"], c["h0"][1:2])
    assert np.array_equal(y[:4, 1:2], part) and not y[4:, 1].any()
    assert np.array_equal(h[1:2], last)


@pytest.mark.parametrize("done,lens", [(False, False), (True, False), (False, True), (True, True)])
def test_gradient_against_differences(done, lens):
    c = _case(6, 3, 2, 3, done, lens)
    g = np.random.default_rng(4)
    dy, dh = g.normal(size=(6, 3, 2)), g.normal(size=(3, 2))

    def loss(**kw):
        y, h = recur.forward(**{**c, **kw})
        return (y * dy).sum() + (h * dh).sum()

    dx, dr, di, dlam, dh0, _ = recur.backward(**c, dy=dy, dh_last=dh)
    eps = 1e-5                          # central differences: error ~ eps^2 = 1e-10 and 1e-16/eps
    for name, grad in (("x", dx), ("r", dr), ("i", di), ("lam", dlam), ("h0", dh0)):
        for at in np.ndindex(*c[name].shape):
            up, down = c[name].copy(), c[name].copy()
            up[at] += eps
            down[at] -= eps
            diff = (loss(**{name: up}) - loss(**{name: down})) / (2 * eps)
            assert abs(diff - grad[at]) < 1e-7 * max(1.0, abs(diff)), (name, at)


def test_closed_gates_have_finite_gradients():
    """L = 0 (a gate of exactly 0): a = 1, beta = 0, and every gradient is finite."""
    c = _case(3, 1, 2, 5)
    c["r"][:] = -800.0
    dx, dr, di, dlam, dh0, _ = recur.backward(**c, dy=np.ones((3, 1, 2)))
    for v in (dx, dr, di, dlam, dh0):
        assert np.isfinite(v).all()
    assert np.array_equal(dh0, np.full((1, 2), 3.0))
