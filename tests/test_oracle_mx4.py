"""Pins of the 4-bit oracle: the format's own tables."""

import numpy as np
import pytest

from oracle import mx4


def _block(*v):
    x = np.zeros((1, 32))
    x[0, :len(v)] = v
    return x


def test_every_code_stands_for_itself():
    x = _block(*mx4.GRID, *-mx4.GRID)
    assert np.array_equal(mx4.values(x), x)


@pytest.mark.parametrize("tie,want", [(0.25, 0), (0.75, 1), (1.25, 1), (1.75, 2), (2.5, 2),
                                      (3.5, 4), (5, 4)])
def test_ties_go_to_the_even_code(tie, want):
    x = mx4.values(_block(4.0, tie, -tie, np.nextafter(tie, 0), np.nextafter(tie, 9)))
    assert x[0, 1] == want and x[0, 2] == -want
    assert x[0, 3] <= want <= x[0, 4] and x[0, 3] < x[0, 4]


def test_the_scale_follows_the_largest_and_the_top_saturates():
    for p in (-20, 0, 7):
        s = 2.0 ** p
        for top, want in ((4.0, 4.0), (5.1, 6.0), (6.0, 6.0), (7.9, 6.0)):
            assert mx4.values(_block(top * s))[0, 0] == want * s
        assert mx4.values(_block(8.0 * s))[0, 0] == 8.0 * s


def test_blocks_are_their_own():
    x = np.concatenate([_block(1.0), _block(1e-6, np.inf), _block(3e38), np.zeros((1, 32))], axis=1)
    q = mx4.values(x)
    assert q[0, 0] == 1.0 and np.isnan(q[0, 32:64]).all() and np.isfinite(q[0, 64:]).all()
    assert not q[0, 96:].any()


def test_the_smallest_scale():
    x = _block(2.0 ** -149, 2.0 ** -127, 1.5 * 2.0 ** -126)
    assert np.array_equal(mx4.values(x)[0, :3], [0.0, 2.0 ** -127, 1.5 * 2.0 ** -126])


def test_relative_error_of_the_largest():
    x = np.random.default_rng(0).normal(size=(64, 320))
    q = mx4.values(x).reshape(64, 10, 32)
    x = x.reshape(64, 10, 32)
    top = np.abs(x).max(axis=2, keepdims=True)
    assert (np.abs(q - x) <= top / 4 + 1e-15).all()
