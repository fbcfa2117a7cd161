"""How exact the gated delta rule's gradients are, beyond what test_gpu_delta.py asks."""

import numpy as np
import pytest
import torch

from gpu_common import say
from oracle import delta
from test_gpu_delta import Case, host

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [32, 64, 128])
def test_bf16_gradients_are_rounded_once(d):
    """dq, dk and dv are the bf16 numbers next to the exact ones, but for few that lie at a border
    between two.  A value moves over a border with the probability |e| / spacing, where the spacing is
    2^-7 of the power of two below the value: of values as N(0, 1), some 12 octaves of which are wider
    apart than e, 128 * 11 |e| in the mean.  Sums of fp32 products (sqrt(144) roundings of 2^-24 a piece,
    two pieces here) have |e| <= 1e-6 of the values' RMS: 1.4e-3.  One operand with two bf16 numbers in
    place of three, 2^-17 / sqrt(3) of it in the mean, would give 5e-3."""
    say(f"[delta numerics] bf16 gradients, heads of {d}")
    c = Case(32, 32, 2, d, d, torch.bfloat16, seed=d)
    saved = c.dc.saved()
    c.forward(saved)
    c.backward(saved)
    want = delta.backward(**c.exact_inputs(), dy=host(c.dy), dh_last=c.dh.astype(np.float64))
    for name, got in zip(("dq", "dk", "dv"), c.parts(c.out)):
        nearest = torch.from_numpy(want[name]).to(torch.bfloat16)
        off = (got.cpu() != nearest).double().mean().item()
        assert off <= 1.4e-3, (name, off)
