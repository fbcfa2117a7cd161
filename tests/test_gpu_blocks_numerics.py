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
