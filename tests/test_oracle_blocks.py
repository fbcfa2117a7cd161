"""The 64-bit oracles of the norms around a block and of the policy loss: gradients against
differences, and against the learner's oracle."""

import numpy as np
import pytest

from oracle import blocks, ppo


def slope(f, x, d, e=1e-6):
    return (f(x + e * d) - f(x - e * d)) / (2 * e)


@pytest.mark.parametrize("parts", [("x", "y", "z", "w_post", "scale", "w_pre"), ("x", "w_pre"),
                                   ("x", "y", "w_post"), ("x", "y", "z"), ("x", "y", "scale", "w_pre")])
@pytest.mark.parametrize("groups", [1, 3])
def test_norm_gradient_against_differences(parts, groups):
    g = np.random.default_rng(0)
    M, D = 4, 12
    a = {k: g.normal(size=(M, D) if k in "xyz" else D) for k in parts}
    dx_out, dn = g.normal(size=(M, D)), g.normal(size=(M, D)) if "w_pre" in parts else None

    def loss(**kw):
        X, n, _ = blocks.norm_forward(**{**a, **kw}, groups=groups)
        return (X * dx_out).sum() + (0.0 if dn is None else (n * dn).sum())

    grad = blocks.norm_backward(**a, groups=groups, dx_out=dx_out, dn=dn)
    for k in parts:
        d = g.normal(size=a[k].shape)
        want = slope(lambda v: loss(**{k: v}), a[k], d)
        assert abs((grad["d" + k] * d).sum() - want) < 1e-7 * (1 + abs(want)), k


def rows(T=5, B=4, n=3, seed=0):
    g = np.random.default_rng(seed)
    mu, ls = g.normal(size=(T, B, n)), g.normal(size=n) * 0.3
    action = mu + np.exp(ls) * g.normal(size=(T, B, n))
    logp = ppo.log_prob(action.reshape(-1, n), mu.reshape(-1, n), ls).reshape(T, B)
    return dict(mu=mu, log_std=ls, action=action, logp=logp + g.normal(size=(T, B)) * 0.3,
                adv=g.normal(size=(T, B)))


@pytest.mark.parametrize("lens", [None, [0, 2, 5, 1]])
def test_policy_gradient_against_differences(lens):
    a = rows()
    g = np.random.default_rng(2)
    kw = dict(mu_ref=a["mu"] + g.normal(size=a["mu"].shape) * 0.2, log_std_ref=a["log_std"] + 0.1,
              lens=lens, clip=(0.2, 0.3), kl=0.7, ent=0.1)
    _, dmu, dls = blocks.policy_loss(**a, **kw)
    for k, grad in (("mu", dmu), ("log_std", dls)):
        d = g.normal(size=a[k].shape)
        want = slope(lambda v: blocks.policy_loss(**{**a, k: v}, **kw)[0][0], a[k], d, 1e-7)
        assert abs((grad * d).sum() - want) < 1e-6, k


def test_policy_loss_is_the_learners():
    """Without KL and with one clip: L_clip, H and their gradient as the learner's oracle has them."""
    a = rows(seed=3)
    n = 3
    stats, dmu, dls = blocks.policy_loss(**a, clip=(0.25, 0.25), ent=0.02)
    dims = (4, 32, 32, n, 32, 32)
    flat = np.zeros(ppo.param_count(*dims))
    p = ppo.unflatten(flat, dims)
    p["log_std"][:] = a["log_std"]
    flatten = lambda x: x.reshape(-1, *x.shape[2:])  # noqa: E731
    p["b3"][:] = a["mu"][0, 0]
    one = {k: v if k == "log_std" else np.broadcast_to(v[:1, :1], v.shape) if k == "mu" else v
           for k, v in a.items()}
    s1, dmu1, dls1 = blocks.policy_loss(**one, clip=(0.25, 0.25), ent=0.02)
    want, grad = ppo.loss_and_grad(flat, dims, np.zeros((20, 4)), flatten(a["action"]),
                                   a["logp"].reshape(-1), a["adv"].reshape(-1), np.zeros(20))
    got = ppo.unflatten(grad, dims)
    assert np.allclose([s1[1], s1[3], s1[4]], [want[0], want[1], want[3]], atol=1e-12)
    assert np.allclose(got["log_std"], dls1) and np.allclose(got["b3"], dmu1.sum((0, 1)))


def test_kl_of_the_same_policy_is_zero():
    a = rows()
    s, _, _ = blocks.policy_loss(**a, mu_ref=a["mu"], log_std_ref=a["log_std"], kl=1.0)
    assert abs(s[2]) < 1e-15


def test_no_rows():
    a = rows()
    s, dmu, dls = blocks.policy_loss(**a, lens=[0] * 4, ent=0.1)
    assert s[5] == 0 and (dmu == 0).all() and np.allclose(dls, -0.1) and np.isfinite(s).all()
