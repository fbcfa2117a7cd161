"""Norms and policy loss beyond what test_gpu_blocks.py asks: bad numbers, far values, many rows."""

import pytest
import torch

from test_gpu_blocks import BOTH, Loss

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
