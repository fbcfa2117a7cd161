"""4-bit blocks in 64 bits (NumPy): the values that a matrix stands for after tp_mx4_quantize.

Blocks of 32 along K; scale 2^e, e = max(floor(log2 of the largest magnitude) - 2, -127); elements
0, 1/2, 1, 3/2, 2, 3, 4, 6 with a sign, nearest, ties to the even code, at most 6.  A block with a
NaN or an infinity is NaN; a block of zeros is zeros.
"""

import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def nearest(m):
    """Indices of the grid's nearest values of m >= 0: the nearer neighbour, ties to the even one."""
    up = np.searchsorted(GRID, m, side="left").clip(0, 7)
    down = np.maximum(up - 1, 0)
    a, b = m - GRID[down], GRID[up] - m
    return np.where(m >= GRID[7], 7, np.where(a < b, down, np.where(b < a, up,
                                                                     np.where(up % 2 == 0, up, down))))


def values(x):
    x = np.asarray(x, np.float64)
    R, K = x.shape
    v = np.zeros((R, -(-K // 32) * 32))
    v[:, :K] = x
    v = v.reshape(R, -1, 32)
    bad = ~np.isfinite(v).all(axis=2, keepdims=True)
    v = np.where(bad, 0.0, v)
    top = np.abs(v).max(axis=2, keepdims=True)
    e = np.maximum(np.frexp(top)[1] - 3, -127)
    scale = np.where(top > 0, np.ldexp(1.0, e), 1.0)
    q = np.copysign(GRID[nearest(np.abs(v) / scale)], v) * scale
    return np.where(bad, np.nan, q).reshape(R, -1)[:, :K]


def product(a, w, bias=None, act=None):
    """act(a w^T + bias) of matrices of values, and what its fp32 rounding scales with."""
    z = a @ w.T
    mass = np.abs(a) @ np.abs(w).T
    if bias is not None:
        z, mass = z + bias, mass + np.abs(bias)
    return (np.tanh(z) if act == "tanh" else z), mass
