"""The delta rule's 64-bit oracle: its gradient against differences, its special cases."""

import numpy as np
import pytest

from oracle import delta


def inputs(T=7, B=3, H=2, dk=5, dv=4, seed=0, done=False, ragged=False):
    g = np.random.default_rng(seed)
    a = dict(q=g.normal(size=(T, B, H, dk)), k=g.normal(size=(T, B, H, dk)),
             v=g.normal(size=(T, B, H, dv)), r=g.normal(size=(T, B, H)),
             b=g.normal(size=(T, B, H)), lam=g.normal(size=H) - 2.0,
             h0=g.normal(size=(B, H, dk, dv)))
    m = dict(done=(g.random((T, B)) < 0.3).astype(np.uint8) if done else None,
             lens=np.array([0, T // 2, T]) if ragged else None)
    return a, m, g.normal(size=(T, B, H, dv)), g.normal(size=(B, H, dk, dv))


@pytest.mark.parametrize("done,ragged", [(False, False), (True, False), (True, True)])
def test_gradient_against_differences(done, ragged):
    a, m, dy, dh = inputs(done=done, ragged=ragged)

    def loss(**kw):
        y, h = delta.forward(**{**a, **kw}, **m)
        return (y * dy).sum() + (h * dh).sum()

    grad = delta.backward(**a, **m, dy=dy, dh_last=dh)
    g = np.random.default_rng(1)
    for name in a:
        d = g.normal(size=a[name].shape)
        e = 1e-6
        want = (loss(**{name: a[name] + e * d}) - loss(**{name: a[name] - e * d})) / (2 * e)
        got = (grad["d" + name] * d).sum()
        assert abs(got - want) < 1e-6 * (1.0 + abs(want)), (name, got, want)


def test_a_sequence_in_two_parts_is_the_whole():
    a, m, _, _ = inputs(T=9)
    y, h = delta.forward(**a)
    first = {n: x[:4] if n not in ("lam", "h0") else x for n, x in a.items()}
    y1, h1 = delta.forward(**first)
    rest = {n: x[4:] if n not in ("lam", "h0") else x for n, x in a.items()}
    y2, h2 = delta.forward(**{**rest, "h0": h1})
    assert np.allclose(np.concatenate([y1, y2]), y, atol=1e-13) and np.allclose(h2, h, atol=1e-13)


def test_an_open_gate_and_a_full_write_recall_the_last_value():
    """beta = 1, no decay: a key reads back what was written to it last."""
    a, _, _, _ = inputs(T=1)
    a["b"] += 60.0
    a["lam"] -= 60.0
    a["q"] = a["k"]
    y, _ = delta.forward(**a)
    length = np.sqrt((a["k"] ** 2).sum(-1) / ((a["k"] ** 2).sum(-1) + delta.EPS))
    assert np.allclose(y, a["v"], atol=3 * (1 - length.min()) * 10 + 1e-12)


def test_masks():
    a, _, dy, dh = inputs(T=6)
    lens = np.array([0, 3, 6])
    y, h = delta.forward(**a, lens=lens)
    assert (y[:, 0] == 0).all() and (y[3:, 1] == 0).all() and np.array_equal(h[0], a["h0"][0])
    grad = delta.backward(**a, lens=lens, dy=dy, dh_last=dh)
    assert (grad["dq"][3:, 1] == 0).all() and np.array_equal(grad["dh0"][0], dh[0])
    done = np.zeros((6, 3), np.uint8)
    done[2] = 1
    y, _ = delta.forward(**a, done=done)
    b = {n: x[3:] if n not in ("lam", "h0") else x for n, x in a.items()}
    y2, _ = delta.forward(**{**b, "h0": None})
    assert np.array_equal(y[3:], y2)
