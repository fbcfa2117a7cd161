"""The norms around a block and the clipped policy loss in 64 bits, by their definitions (NumPy)."""

import numpy as np

LN_2PI = 1.8378770664093453


def _sigmoid(x):
    e = np.exp(-np.abs(x))
    return np.where(x >= 0, 1.0 / (1.0 + e), e / (1.0 + e))


def _grouped(x, groups):
    return x.reshape(x.shape[0], groups, -1)


def norm_forward(x, y=None, z=None, w_post=None, scale=None, w_pre=None, groups=1, eps=1e-6):
    """X and n (None without w_pre); what the gradient needs comes along."""
    f = yn = ry = None
    X = np.array(x, np.float64)
    if y is not None:
        yn = np.array(y, np.float64)
        if w_post is not None:
            g = _grouped(yn, groups)
            ry = 1.0 / np.sqrt((g * g).mean(2, keepdims=True) + eps)
            yn = (g * ry).reshape(yn.shape)
        f = yn * (1.0 if w_post is None else w_post) * (1.0 if z is None else z * _sigmoid(z))
        X = X + (1.0 if scale is None else scale) * f
    rx = 1.0 / np.sqrt((X * X).mean(1, keepdims=True) + eps)
    return X, None if w_pre is None else X * rx * w_pre, (f, yn, ry, rx)


def norm_backward(x, y=None, z=None, w_post=None, scale=None, w_pre=None, groups=1, eps=1e-6,
                  dx_out=None, dn=None):
    """Gradients of sum(X dx_out) + sum(n dn); with `_size` after its name, what the rounding of each
    scales with: its terms' magnitudes, X's among them (x and what is added may cancel)."""
    X, _, (f, yn, ry, rx) = norm_forward(x, y, z, w_post, scale, w_pre, groups, eps)
    dX = np.zeros_like(X) if dx_out is None else np.array(dx_out, np.float64)
    one = lambda w: 1.0 if w is None else w  # noqa: E731
    xs = rx * (np.abs(x) + (0.0 if f is None else np.abs(one(scale) * f)))
    grow = np.sqrt((xs * xs).mean(1, keepdims=True))
    size = np.abs(dX)
    out = dict(x_size=xs / rx)
    if dn is not None:
        t, xn = dn * w_pre, X * rx
        out["n_size"] = xs * np.abs(w_pre) * grow
        out["dw_pre"], out["dw_pre_size"] = (dn * xn).sum(0), (np.abs(dn) * xs * grow).sum(0)
        dX = dX + rx * (t - xn * (t * xn).mean(1, keepdims=True))
        size = size + rx * grow * (np.abs(t) + xs * (np.abs(t) * xs).mean(1, keepdims=True))
    out["dx"], out["dx_size"] = dX, size
    if y is None:
        return out
    if scale is not None:
        out["dscale"], out["dscale_size"] = (dX * f).sum(0), (size * np.abs(f)).sum(0)
    df, size = dX * one(scale), size * np.abs(one(scale))
    w = one(w_post)
    gate = 1.0
    if z is not None:
        s = _sigmoid(z)
        gate = z * s
        out["dz"] = df * yn * w * s * (1.0 + z * (1.0 - s))
        out["dz_size"] = size * np.abs(yn * w) * s * (1.0 + np.abs(z) * (1.0 - s))
    d, ds = df * w * gate, size * np.abs(w * gate)
    if w_post is not None:
        out["dw_post"] = (df * yn * gate).sum(0)
        out["dw_post_size"] = (size * np.abs(yn * gate)).sum(0)
        dg, yg, sg = _grouped(d, groups), _grouped(yn, groups), _grouped(ds, groups)
        d = (ry * (dg - yg * (dg * yg).mean(2, keepdims=True))).reshape(d.shape)
        ds = (ry * (sg + np.abs(yg) * (sg * np.abs(yg)).mean(2, keepdims=True))).reshape(d.shape)
    out["dy"], out["dy_size"] = d, ds
    return out


def policy_loss(mu, log_std, action, logp, adv, mu_ref=None, log_std_ref=None, lens=None,
                clip=(0.2, 0.2), kl=0.0, ent=0.0):
    """stats [6] (loss, policy term, mean KL, entropy, clip fraction, rows), dmu, dlog_std."""
    T, B, n = mu.shape
    on = np.ones((T, B), bool)
    if lens is not None:
        on = np.arange(T)[:, None] < np.asarray(lens)[None]
    N = int(on.sum())
    sigma = np.exp(log_std)
    H = float((log_std + 0.5 * (1.0 + LN_2PI)).sum())
    dmu, dls = np.zeros((T, B, n)), np.full(n, -ent)
    if N == 0:
        return np.array([-ent * H, 0.0, 0.0, H, 0.0, 0.0]), dmu, dls
    z = (action[on] - mu[on]) / sigma
    lp = (-0.5 * z * z - log_std).sum(1) - 0.5 * n * LN_2PI
    rho = np.exp(lp - logp[on])
    A = adv[on]
    held = np.minimum(np.maximum(rho, 1.0 - clip[0]), 1.0 + clip[1])
    free = rho * A <= held * A
    policy = -np.where(free, rho * A, held * A).mean()
    w = np.where(free, -rho * A / N, 0.0)[:, None]
    d, g = w * z / sigma, w * (z * z - 1.0)
    KL = 0.0
    if mu_ref is not None:
        o = (mu[on] - mu_ref[on]) / sigma
        s2 = np.exp(2.0 * (log_std_ref - log_std))
        KL = float((log_std - log_std_ref - 0.5 + 0.5 * s2 + 0.5 * o * o).sum(1).mean())
        d, g = d + kl / N * o / sigma, g + kl / N * (1.0 - s2 - o * o)
    dmu[on] = d
    dls = dls + g.sum(0)
    out = float(((rho < 1.0 - clip[0]) | (rho > 1.0 + clip[1])).mean())
    return np.array([policy + kl * KL - ent * H, policy, KL, H, out, N]), dmu, dls
