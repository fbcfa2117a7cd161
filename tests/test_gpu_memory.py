"""The memory layer: 4-bit product and recurrence together, on a rollout's stored observations."""

import numpy as np
import pytest
import torch

import workloads as W
from gpu_common import build_problem
from oracle import mx4, recur
from paper_2111_05188_amd import memory, tp

pytestmark = pytest.mark.gpu


def host(t):
    return t.double().cpu().numpy()


def rms_close(got, want, tol):
    got, want = host(got), np.asarray(want)
    assert np.abs(got - want).max() <= tol * max(np.sqrt(np.mean(want ** 2)), np.abs(want).max())


def test_layer_on_a_rollouts_trajectory():
    """encode over the stored rows of a rollout, its gradients, and the same bars step by step."""
    cfg = W.get_config("tiny")
    pb, _ = build_problem(cfg, W.make_market(cfg), W.make_t0(cfg))
    pb.set_values(W.make_values(cfg))
    pb.step(7)
    obs, done = pb.traj.obs, pb.traj.done
    T, B, ld = obs.shape
    layer = memory.MemoryLayer.init(cfg.S, 48, 1, torch.float32)
    y, last = layer.encode(obs, done)
    g = torch.Generator("cuda").manual_seed(2)
    dy = torch.randn(T, B, 48, generator=g, device="cuda")
    dW, dlam, dh0 = layer.gradients(dy)
    torch.cuda.synchronize()
    # the same in 64 bits: values of the 4-bit operands, then the definition, on some envs
    w = mx4.values(host(layer.W))
    x = mx4.values(host(obs.reshape(T * B, ld)[:, :cfg.S]))
    gates = (x @ w.T).reshape(T, B, -1)
    # fp32 sums of 31 products, then 2e-5 of the recurrence
    rms_close(layer.gates, gates, 1e-6)
    pick = [0, 5, B - 1]
    parts = [gates[:, pick, k * 48:(k + 1) * 48] for k in range(3)]
    lam = host(layer.lam)
    d = host(done)[:, pick]
    wy, wl = recur.forward(*parts, lam, None, d)
    rms_close(y[:, pick], wy, 3e-5)
    rms_close(last[pick], wl, 3e-5)
    dx, dr, di, _, _, _ = recur.backward(*parts, lam, host(dy)[:, pick], None, None, d)
    rms_close(layer.dgates[:, pick], np.concatenate([dx, dr, di], axis=2), 3e-5)
    # W's gradient: the product of both operands' 4-bit values along the rows
    a = mx4.values(host(layer.dgates.reshape(T * B, -1)).T)
    b = mx4.values(host(obs.reshape(T * B, ld)[:, :cfg.S]).T)
    want, mass = mx4.product(a, b)
    assert (np.abs(host(dW) - want) <= (T * B / 64 + 8) * 2.0 ** -23 * mass).all()
    # bar by bar
    h = torch.zeros(B, 48, device="cuda")
    for t in range(20):
        yt = layer.step(obs[t], h, done[t].contiguous())
        torch.cuda.synchronize()
        rms_close(yt, host(y[t]), 2e-5)


def test_layer_learns_to_remember():
    """Below half of what knowing nothing (1.0) leaves."""
    losses = memory.train_to_remember()
    assert losses[0] > 1.0 and losses[-1] < 0.5, losses[::50]


def test_updates_reach_the_4_bit_weights():
    layer = memory.MemoryLayer.init(31, 16, 3, torch.float32)
    obs = torch.randn(10, 4, 32, generator=torch.Generator("cuda").manual_seed(4), device="cuda")
    y0 = layer.encode(obs)[0].clone()
    dW, dlam, _ = layer.gradients(torch.ones(10, 4, 16, device="cuda"))
    layer.W.add_(dW, alpha=-0.1)
    layer.lam.add_(dlam, alpha=-0.1)
    layer.refresh()
    y1 = layer.encode(obs)[0]
    torch.cuda.synchronize()
    assert float(y1.sum()) < float(y0.sum())
    back = torch.empty(48, 31, device="cuda")
    tp.mx4_dequantize(layer.w4, back)
    torch.cuda.synchronize()
    assert np.array_equal(host(back), mx4.values(host(layer.W)))


@pytest.mark.parametrize("dtype,tol", [(torch.float32, 2e-5), (torch.bfloat16, 2e-5 + 2.0 ** -8)])
def test_a_trajectory_in_parts(dtype, tol):
    """The last states of one encode are the first of the next, as they were returned."""
    layer = memory.MemoryLayer.init(31, 64, 5, dtype)
    obs = torch.randn(1200, 2, 32, generator=torch.Generator("cuda").manual_seed(6), device="cuda")
    y, last = (t.clone() for t in layer.encode(obs))
    h, parts = None, []
    for k in range(3):
        out, h = layer.encode(obs[400 * k:400 * (k + 1)], h0=h)
        parts.append(out.clone())
    torch.cuda.synchronize()
    rms_close(torch.cat(parts), host(y), tol)
    rms_close(h, host(last), 2e-5)
