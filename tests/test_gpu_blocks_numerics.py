"""Norms and policy loss beyond what test_gpu_blocks.py asks: bad numbers, far values, many rows."""

import numpy as np
import pytest
import torch

from oracle import blocks
from paper_2111_05188_amd import tp
from test_gpu_blocks import BOTH, Loss, Norm, host

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("what", ["adv", "logp", "action", "mu_ref"])
def test_a_bad_row_of_the_loss_shows_in_its_gradient(what, dtype):
    """A NaN among what a row reads is in the loss, in its means' gradient and in log_std's; the other
    rows' gradients are as without it."""
    c = Loss(4, 6, 30, dtype, seed=5)
    _, want, _ = c.run()
    t = c.t[what]
    t[(3, 2) if t.dim() == 2 else (3, 2, slice(None))] = float("nan")
    stats, dmu, dls = c.run()
    assert torch.isnan(stats[0]) and torch.isnan(dmu[3, 2]).all() and torch.isnan(dls).all()
    other = torch.ones(4, 6, dtype=torch.bool, device="cuda")
    other[3, 2] = False
    assert torch.equal(dmu[other], want[other])


@pytest.mark.parametrize("dtype", BOTH)
def test_a_ratio_past_every_number_without_an_advantage(dtype):
    """It is clipped, and adds nothing."""
    c = Loss(4, 6, 30, dtype, seed=6)
    c.t["logp"][1, 1] -= 2000.0
    c.t["adv"][1, 1] = 0.0
    c.kw["kl"], c.ls_ref, c.t["mu_ref"] = 0.0, None, None
    c.setup()
    stats, dmu, dls = c.run()
    assert torch.isfinite(stats).all() and torch.isfinite(dls).all() and (dmu[1, 1] == 0).all()


@pytest.mark.parametrize("D", [64, 63])
def test_gates_far_from_zero(D):
    """The gate's own relative error does not grow with its pre-activation, -80 to 80.  Of f, in half
    steps of 2^-24: the row's sum, sqrt(D) of them halved by the root, 4; its root 2; the exponential 2,
    its factor 2, its sum 1, the quotient 1; five products 5: 17.  Of dz four products and two sums more:
    23 of its terms.  (1e-36: smaller ones have fewer bits.)"""
    c = Norm(40, D, 1, torch.float32, parts=("x", "y", "z", "w_post", "scale"), seed=D)
    c.t["x"].zero_()
    c.t["z"].copy_(torch.linspace(-80.0, 80.0, 40 * D).view(D, 40).t())
    new = [c.new() for _ in range(4)]
    tp.norm_forward(c.nc, c.t["x"], c.t["y"], c.t["z"], new[0], None)
    tp.norm_backward(c.nc, c.t["x"], c.t["y"], c.t["z"], c.t["dx_out"], None, *new[1:], None, None, None,
                     c.nc.workspace())
    X, _, _ = blocks.norm_forward(**c.exact())
    err = np.abs(host(new[0]) - X) / (np.abs(X) + 1e-36)
    assert err.max() <= 17 * 2.0 ** -24, err.max() * 2 ** 24
    want = blocks.norm_backward(**c.exact(), dx_out=host(c.t["dx_out"]))
    err = np.abs(host(new[3]) - want["dz"]) / (want["dz_size"] + 1e-36)
    assert err.max() <= 23 * 2.0 ** -24, err.max() * 2 ** 24


@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("M,D", [(1 << 20, 513), (1 << 24, 8)])
def test_weights_gradients_of_many_rows(M, D, dtype):
    """Of rows all alike, as many times one's, whatever their number.  Half steps of 2^-24 in a row's
    terms: x (of ones) squared and added up none, their mean, root and product with x 4, with dn 1, f's
    5 more; sums of 32 of them 32 in fp32 at most, 2^-24 each of the largest partial sum: 42 in all, of
    which equal terms' sums, that round alike, may use up any number; 64-bit sums of the rest none.  The
    result's own rounding 1."""
    g = torch.Generator("cuda").manual_seed(D)
    rows = lambda v: v.to(dtype).expand(M, D).contiguous()  # noqa: E731
    vec = lambda: torch.rand(D, generator=g, device="cuda") + 0.5  # noqa: E731
    x, y, dn, dx_out = torch.ones(D, device="cuda"), torch.zeros(D, device="cuda"), vec(), vec()
    y[::2] = 1.0
    w_pre, w_post, scale = vec(), vec(), vec()
    nc = tp.NormT(M, D, dtype, w_pre=w_pre, w_post=w_post, scale=scale)
    out = [torch.empty(M, D, dtype=dtype, device="cuda") for _ in range(2)]
    dw = [torch.empty(D, device="cuda") for _ in range(3)]
    tp.norm_backward(nc, rows(x), rows(y), None, rows(dx_out), rows(dn), *out, None, *dw, nc.workspace())
    one = lambda v: host(v.to(dtype))[None]  # noqa: E731
    want = blocks.norm_backward(one(x), one(y), w_post=host(w_post), scale=host(scale), w_pre=host(w_pre),
                                dx_out=one(dx_out), dn=one(dn))
    for got, k in zip(dw, ("dw_post", "dscale", "dw_pre")):
        err = np.abs(host(got) - M * want[k]) / (M * want[k + "_size"] + 1e-30)
        assert err.max() <= 43 * 2.0 ** -24, (k, err.max() * 2 ** 24)


@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("D", [128, 301])
def test_outputs_in_the_inputs_places_and_between_their_rows(D, dtype):
    """An output in any input's buffer, and arrays side by side in one buffer's rows, whole or with other
    pitches one after the other."""
    c = Norm(300, D, 1, dtype, seed=7)
    X, n = c.forward()
    want = c.backward()
    t = {k: v.clone() for k, v in c.t.items()}
    tp.norm_forward(c.nc, t["x"], t["y"], t["z"], t["z"], t["y"])
    assert torch.equal(t["z"], X) and torch.equal(t["y"], n)
    t = {k: v.clone() for k, v in c.t.items()}
    dw = [torch.empty(D, device="cuda") for _ in range(3)]
    tp.norm_backward(c.nc, t["x"], t["y"], t["z"], t["dx_out"], t["dn"], t["dn"], t["y"], t["z"], *dw,
                     c.nc.workspace())
    assert all(torch.equal(t[a], want[b]) for a, b in (("dn", "dx"), ("y", "dy"), ("z", "dz")))
    assert all(torch.equal(a, want[b]) for a, b in zip(dw, ("dw_post", "dscale", "dw_pre")))
    wide = torch.empty(300, 5 * D, dtype=dtype, device="cuda")
    part = [wide[:, i * D:(i + 1) * D] for i in range(5)]
    for p, k in zip(part, "xyz"):
        p.copy_(c.t[k])
    tp.norm_forward(c.nc, *part)
    assert torch.equal(part[3], X) and torch.equal(part[4], n)
    flat = torch.empty(300 * 3 * D, dtype=dtype, device="cuda")
    a, b = flat[:300 * D].view(300, D), flat[300 * D:].view(300, 2 * D)[:, D:]
    tp.norm_forward(c.nc, c.t["x"], c.t["y"], c.t["z"], a, b)
    assert torch.equal(a, X) and torch.equal(b, n)
