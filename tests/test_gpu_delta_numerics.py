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


def check_decays(c):
    """r's and lambda's gradients against what passes a step's decay, D and e^g S, alone: however strong
    the decay, their products' errors are those of the two, 2e-5 (test_gpu_delta.py), and of the decays,
    2^-23 of a sum of log-decays.  An error of a state stays for the memory's M steps, so that lambda's,
    a sum over steps, has sqrt(M) of what single ones would add: 7e-7 sqrt(M / 16) sqrt(M) times 2.5
    sigma, 4.4e-7 M.  (1e-35: what fp32 has no numbers for.)"""
    saved = c.dc.saved()
    c.forward(saved)
    dlam, _ = c.backward(saved)
    want = delta.backward(**c.exact_inputs(), dy=host(c.dy), dh_last=c.dh.astype(np.float64))
    rate = 8.0 * delta.softplus(c.lam.astype(np.float64))
    own = rate * 2.0 ** -23
    half = 2.0 ** -8 if c.dtype == torch.bfloat16 else 2.0 ** -22
    bound = half * np.abs(want["dr"]) + (2e-5 + own) * want["dr_across"] + 1e-35
    over = np.abs(host(c.parts(c.out)[3]) - want["dr"]) / bound
    assert over.max() <= 1.0, ("dr", over.max(), np.median(over), (over > 1).mean())
    memory = np.minimum(c.T, 1.0 / -np.expm1(-rate / 2.0))
    bound = 2.0 ** -22 * np.abs(want["dlam"]) + (np.maximum(2e-5, 4.4e-7 * memory) + own) * want["dlam_across"]
    over = np.abs(host(dlam) - want["dlam"]) / (bound + 1e-35)
    assert over.max() <= 1.0, ("dlam", over, host(dlam), want["dlam"])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shape", [(1, 2, 2, 64, 64), (33, 3, 2, 64, 64), (70, 2, 3, 32, 20), (50, 2, 2, 100, 128),
                                   (20, 40, 8, 64, 64), (700, 1, 2, 64, 48), (3300, 1, 1, 32, 32)])
@pytest.mark.parametrize("lam", [None, 0.0, 3.0, 6.0, 10.0, 30.0])
def test_gradients_of_decays_of_any_strength(shape, lam, dtype):
    """From memories of 10 to 2,000 bars (None) to ones of less than a bar."""
    say(f"[delta numerics] decays {shape} {lam} {dtype}")
    c = Case(*shape, dtype, 0.02, True, seed=sum(shape))
    if lam is not None:
        c.lam[:] = lam
    if c.B == 1:
        c.lens[0] = c.T
    c.setup()
    check_decays(c)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shape", [(40, 4, 3, 64, 64), (2000, 1, 2, 32, 32)])
@pytest.mark.parametrize("where", range(4))
def test_a_part_that_dominates(shape, where, dtype):
    """A quarter of the sequences, or of one's steps, whose values are 32 times the others': lambda's
    gradient is nearly all from there."""
    c = Case(*shape, dtype, seed=where)
    v = c.parts(c.rows)[2]
    n = max(c.B, c.T if c.B == 1 else 0) // 4
    part = v[:, where * n:(where + 1) * n] if c.B > 1 else v[where * n:(where + 1) * n]
    part *= 32.0
    check_decays(c)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_bad_number_reaches_no_decay_before_it(dtype):
    """A NaN among the values: r's gradients of the steps before it, to the step, are as without it."""
    c = Case(90, 1, 2, 64, 64, dtype, seed=4)

    def run():
        saved = c.dc.saved()
        c.forward(saved)
        c.backward(saved)
        return host(c.parts(c.out)[3])

    fine = run()
    c.parts(c.rows)[2][77, 0, 1, 5] = float("nan")
    got = run()
    want = delta.backward(**c.exact_inputs(), dy=host(c.dy), dh_last=c.dh.astype(np.float64))
    assert np.isfinite(got[:78]).all() and np.isfinite(got[:, :, 0]).all()
    assert np.isnan(got[78:, 0, 1]).all()
    half = 2.0 ** -7 if dtype == torch.bfloat16 else 2.0 ** -21
    bound = half * np.abs(fine) + 4e-5 * want["dr_across"]
    assert (np.abs(got - fine) <= bound)[:78].all() and (np.abs(got - fine) <= bound)[:, :, 0].all()
