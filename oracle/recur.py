"""Gated linear recurrence in 64 bits, by its definition, one step at a time (NumPy).

  rho = sigmoid(r), iota = sigmoid(i), L = -8 softplus(lambda) rho, a = exp(L),
  beta = sqrt(1 - a^2), h_t = a h_{t-1} + beta iota x, y_t = h_t;
  h := 0 after a step with done set; steps past a sequence's length leave h as it is.
"""

import numpy as np


def sigmoid(x):
    e = np.exp(-np.abs(x))
    return np.where(x >= 0, 1.0 / (1.0 + e), e / (1.0 + e))


def softplus(x):
    return np.maximum(x, 0.0) + np.log1p(np.exp(-np.abs(x)))


def coefficients(x, r, i, lam):
    """L, a, beta, iota, rho of one step ([B][D])."""
    rho, iota = sigmoid(r), sigmoid(i)
    L = -8.0 * softplus(lam) * rho
    return L, np.exp(L), np.sqrt(-np.expm1(2.0 * L)), iota, rho


def forward(x, r, i, lam, h0=None, done=None, lens=None):
    """y [T][B][D] and the last states [B][D]."""
    T, B, D = x.shape
    h = np.zeros((B, D)) if h0 is None else np.array(h0, np.float64)
    y = np.zeros((T, B, D))
    for t in range(T):
        for b in range(B):
            if lens is not None and t >= lens[b]:
                continue
            _, a, beta, iota, _ = coefficients(x[t, b], r[t, b], i[t, b], lam)
            h[b] = a * h[b] + beta * (iota * x[t, b])
            y[t, b] = h[b]
            if done is not None and done[t, b]:
                h[b] = 0.0
    return y, h


def backward(x, r, i, lam, dy, dh_last=None, h0=None, done=None, lens=None):
    """Gradients of sum(y dy) + sum(h_last dh_last): dx, dr, di, dlam, dh0, and sum |w| of
    lambda's sum (what its rounding scales with)."""
    T, B, D = x.shape
    y, _ = forward(x, r, i, lam, h0, done, lens)
    dx, dr, di = np.zeros_like(y), np.zeros_like(y), np.zeros_like(y)
    G = np.zeros((B, D)) if dh_last is None else np.array(dh_last, np.float64)
    dlam, mass = np.zeros(D), np.zeros(D)
    kappa = sigmoid(lam) / softplus(lam)
    for t in reversed(range(T)):
        for b in range(B):
            if lens is not None and t >= lens[b]:
                continue
            if done is not None and done[t, b]:
                G[b] = 0.0
            if t == 0:
                prev = np.zeros(D) if h0 is None else h0[b]
            else:
                prev = np.zeros(D) if done is not None and done[t - 1, b] else y[t - 1, b]
            L, a, beta, iota, rho = coefficients(x[t, b], r[t, b], i[t, b], lam)
            g = dy[t, b] + G[b]
            q = iota * x[t, b]
            ratio = np.where(beta > 0, L / np.where(beta > 0, beta, 1.0), 0.0)
            w = g * (L * a * prev - q * a * a * ratio)
            dx[t, b] = g * beta * iota
            di[t, b] = g * beta * q * (1.0 - iota)
            dr[t, b] = w * (1.0 - rho)
            dlam += kappa * w
            mass += kappa * np.abs(w)
            G[b] = a * g
    return dx, dr, di, dlam, G, mass
