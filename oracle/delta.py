"""Gated delta rule in 64 bits, by its definition, one step at a time (NumPy).

  q^ = q / sqrt(q.q + 1e-6), k^ likewise, g = -8 softplus(lambda) sigmoid(r), beta = sigmoid(b),
  S' = e^g S, u = beta (v - S'^T k^), S = S' + k^ u^T, y = S^T q^;
  S := 0 after a step with done set; steps past a sequence's length leave S as it is.
"""

import numpy as np

from .recur import sigmoid, softplus

EPS = 1e-6
AHEAD = 32          # steps that dr_mass adds up


def _unit(x):
    return x / np.sqrt((x * x).sum(-1, keepdims=True) + EPS)


def _step(q, k, v, r, b, lam, S):
    """One step of [B][H]; what the gradient needs comes along."""
    q, k = _unit(q), _unit(k)
    g, beta = -8.0 * softplus(lam) * sigmoid(r), sigmoid(b)
    S1 = np.exp(g)[..., None, None] * S
    e = v - np.matmul(k[..., None, :], S1)[..., 0, :]
    u = beta[..., None] * e
    S2 = S1 + k[..., :, None] * u[..., None, :]
    y = np.matmul(q[..., None, :], S2)[..., 0, :]
    return S2, y, (q, k, g, beta, S1, e, u)


def _gates(t, B, done, lens):
    live = np.ones(B, bool) if lens is None else t < np.asarray(lens)
    ends = np.zeros(B, bool) if done is None else live & (np.asarray(done[t]) != 0)
    return live, ends


def forward(q, k, v, r, b, lam, h0=None, done=None, lens=None, states=None):
    """y [T][B][H][dv] and the last states [B][H][dk][dv]; states: a list that gets those before
    each step."""
    T, B, H, dk = q.shape
    dv = v.shape[3]
    S = np.zeros((B, H, dk, dv)) if h0 is None else np.array(h0, np.float64)
    y = np.zeros((T, B, H, dv))
    for t in range(T):
        if states is not None:
            states.append(S.copy())
        live, ends = _gates(t, B, done, lens)
        S2, yt, _ = _step(q[t], k[t], v[t], r[t], b[t], lam, S)
        y[t][live] = yt[live]
        S = np.where(live[:, None, None, None], S2, S)
        S[ends] = 0.0
    return y, S


def backward(q, k, v, r, b, lam, dy, dh_last=None, h0=None, done=None, lens=None):
    """Gradients of sum(y dy) + sum(h_last dh_last): dq, dk, dv, dr, db, dlam, dh0; and what the
    roundings of dr [T][B][H] and dlam [H] scale with, the lengths of the vectors whose products
    add up to them, and of dq and dk, the gradients of the unit rows over the rows' lengths.
    dr_across [T][B][H], dlam_across [H]: the same of dr and dlam, with only what passes a step's decay:
    |e^g S| |D| / sqrt(d) of e^g S and its gradient D, whose product the gradient of g is (roundings of
    single elements, in states of rank one at least)."""
    T, B, H, dk = q.shape
    states = []
    forward(q, k, v, r, b, lam, h0, done, lens, states)
    G = np.zeros_like(states[0]) if dh_last is None else np.array(dh_last, np.float64)
    dq, dk_, dv, dr, db = (np.zeros_like(x) for x in (q, k, v, r, b))
    dlam, w = np.zeros(H), np.zeros(r.shape)
    sizes = dict(dq_size=np.ones(r.shape + (1,)), dk_size=np.ones(r.shape + (1,)))
    size, shut, across, past = (np.zeros(r.shape) for _ in range(4))
    norm = lambda x: np.sqrt((x * x).sum(-1))  # noqa: E731
    for t in reversed(range(T)):
        live, ends = _gates(t, B, done, lens)
        G[ends] = 0.0
        S2, _, (qn, kn, g, beta, S1, e, u) = _step(q[t], k[t], v[t], r[t], b[t], lam, states[t])
        D2 = G + qn[..., :, None] * dy[t][..., None, :]
        dqn = np.matmul(S2, dy[t][..., None])[..., 0]
        du = np.matmul(kn[..., None, :], D2)[..., 0, :]
        de = beta[..., None] * du
        D1 = D2 - kn[..., :, None] * de[..., None, :]
        dkn = np.matmul(D2, u[..., None])[..., 0] - np.matmul(S1, de[..., None])[..., 0]
        dg = (D1 * S1).sum((-2, -1))
        m = live
        for name, out, x, n, d in (("dq_size", dq, q[t], qn, dqn), ("dk_size", dk_, k[t], kn, dkn)):
            length = np.sqrt((x * x).sum(-1, keepdims=True) + EPS)
            sizes[name][t] = np.maximum(1.0, norm(d)[..., None]) / length
            out[t][m] = ((d - n * (n * d).sum(-1, keepdims=True)) / length)[m]
        dv[t][m] = de[m]
        rest, less = sigmoid(-r[t]), sigmoid(-b[t])     # 1 - sigmoid, without cancellation
        w[t][m] = (dg * g)[m]
        dr[t][m] = (dg * g * rest)[m]
        db[t][m] = ((du * e).sum(-1) * beta * less)[m]
        shut[t][m] = (-g * rest)[m]
        past[t][m] = (-g * np.sqrt((D1 * D1).sum((-2, -1)) * (S1 * S1).sum((-2, -1)) / min(dk, v.shape[3])))[m]
        across[t][m] = (past[t] * rest)[m]
        size[t][m] = (norm(dqn) + norm(dkn) + 2.0 * norm(du) * norm(u)
                      + np.sqrt((G * G).sum((-2, -1)) * (S2 * S2).sum((-2, -1))))[m]
        dlam += w[t].sum(0)
        G = np.where(live[:, None, None, None], np.exp(g)[..., None, None] * D1, G)
    kappa = sigmoid(lam) / softplus(lam)
    ahead = np.zeros_like(size)
    for t in range(T):
        ahead[t] = size[t:t + AHEAD].sum(0)
    mass = (ahead * -8.0 * softplus(lam) * -sigmoid(r)).sum((0, 1)) * kappa
    return dict(dq=dq, dk=dk_, dv=dv, dr=dr, db=db, dlam=kappa * dlam, dh0=G,
                dr_mass=ahead * shut, dlam_mass=mass, dr_across=across,
                dlam_across=kappa * np.sqrt((past * past).sum((0, 1))), **sizes)
