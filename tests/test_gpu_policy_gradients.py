"""MatrixPolicy.gradients call by call, down to the embedding: each call's results against the 64-bit
oracle on the inputs it got, and that these are the results of the calls before it."""

import numpy as np
import pytest
import torch

from oracle import blocks, delta
from paper_2111_05188_amd import policy, tp
from test_gpu_policy import host, near, product

pytestmark = pytest.mark.gpu


def spied(monkeypatch, owner, name):
    """The arguments and the result of every call, in order."""
    calls, real = [], getattr(owner, name)

    def call(*args, **kw):
        out = real(*args, **kw)
        calls.append((args, kw, out))
        return out

    monkeypatch.setattr(owner, name, call)
    return calls


def same(a, b):
    return a is b or (a is not None and b is not None and a.data_ptr() == b.data_ptr()
                      and a.numel() == b.numel() and a.dtype == b.dtype)


def setup(dtype, blocks_, T=40, B=16, S=31, n=5, H=2, d=32):
    g = torch.Generator("cuda").manual_seed(6)
    pol = policy.MatrixPolicy(S, n, H=H, d=d, blocks=blocks_, dtype=dtype, seed=5)
    for k, p in pol.parameters().items():       # (no two blocks or channels alike)
        if k.endswith(("w_pre", "w_post", "scale", "w_out")):
            p += 0.3 * torch.randn(p.shape, generator=g, device="cuda")
    obs = torch.randn(T, B, 32, generator=g, device="cuda").to(dtype)
    done = (torch.rand(T, B, generator=g, device="cuda") < 0.05).byte()
    dmu = torch.randn(T, B, n, generator=g, device="cuda").to(dtype)
    return pol, obs, done, dmu, torch.randn(n, generator=g, device="cuda")


@pytest.mark.parametrize("dtype,tol", [(torch.float32, 3e-5), (torch.bfloat16, 3e-5 + 2.0 ** -8)])
def test_every_gradient_on_what_its_call_got(dtype, tol, monkeypatch):
    pol, obs, done, dmu, dls = setup(dtype, 3)
    T, B = done.shape
    M, D = T * B, pol.D
    pol.forward(obs, done)
    norms, deltas = spied(monkeypatch, tp, "norm_backward"), spied(monkeypatch, tp, "delta_backward")
    products = spied(monkeypatch, policy.Matrix, "gradients")
    grads = pol.gradients(dmu, dls)
    torch.cuda.synchronize()
    assert (len(norms), len(deltas), len(products)) == (4, 3, 5)
    assert torch.equal(grads["log_std"], dls)
    near(grads["bias"], host(dmu).reshape(M, -1).sum(0), 1e-5)

    def matrix(m, x, dy, dW):
        """The next product's gradients: of matrix m, input x, output gradient dy."""
        (got_m, got_x, got_dy), kw, (_, dx) = products.pop(0)
        assert got_m is m and same(got_x, x) and same(got_dy, dy)
        near(dW, product(host(dy).T, host(x).T), 1e-4)
        if dx is not None:
            near(dx, product(host(dy), host(m.W).T), tol)
        return dx

    dn, dx = matrix(pol.head, pol.last, dmu.view(M, -1), grads["head"]), None
    tight = []
    for i in (2, 1, 0):
        b, (_, x, n, p, y, _) = pol.blocks[i], pol.kept[i]
        (_, gx, gy, gz, gdx_out, gdn, dx_in, dy, dz, *_), _, _ = norms.pop(0)
        parts, z = b.parts(p.view(T, B, -1))
        assert same(gx, x) and same(gy, y) and same(gz, z) and same(gdx_out, dx) and same(gdn, dn)
        after, name = (pol.w_out, "w_out") if i == 2 else (pol.blocks[i + 1].w_pre, f"{i + 1}.w_pre")
        want = blocks.norm_backward(host(x), host(y).reshape(M, D), host(z).reshape(M, D), host(b.w_post),
                                    host(b.scale), host(after), groups=b.H, dn=host(dn),
                                    dx_out=None if dx is None else host(dx))
        near(dx_in, want["dx"], tol)
        near(dy.reshape(M, D), want["dy"], tol)
        for k, w in ((f"{i}.w_post", "dw_post"), (f"{i}.scale", "dscale"), (name, "dw_pre")):
            near(grads[k], want[w], 1e-4)
        # the block's product gets dq, dk, dv, dz, dr, db side by side
        dp = products[0][0][2]
        args, kw, _ = deltas.pop(0)
        assert same(args[7], dy) and all(same(a, c) for a, c in zip(args[1:6], parts)) and not kw
        wd = delta.backward(*(host(t) for t in parts), host(b.lam), dy=host(dy).reshape(T, B, b.H, b.d),
                            done=host(done))
        side = [wd[k].reshape(M, D) for k in ("dq", "dk", "dv")] + [want["dz"]] + \
               [wd[k].reshape(M, b.H) for k in ("dr", "db")]
        at = np.cumsum([0] + [s.shape[1] for s in side])
        assert at[-1] == dp.shape[1] and same(dz, dp.view(T, B, -1)[..., 3 * D:4 * D])
        for s, u, v in zip(side, at, at[1:]):
            near(dp[:, u:v], s, tol)
        # (per head: 2e-5 of the products that pass a decay, on the dy that the kernel got)
        err = np.abs(host(grads[f"{i}.lam"]) - wd["dlam"])
        assert (err <= 2e-5 * wd["dlam_across"] + 2.0 ** -22 * np.abs(wd["dlam"])).all(), (err, wd["dlam"])
        tight += list(2e-5 * wd["dlam_across"] < 0.01 * np.abs(wd["dlam"]))
        dn, dx = matrix(b.m, n, dp, grads[f"{i}.W"]), dx_in
    (_, gx, gy, gz, gdx_out, gdn, dx_in, *_), _, _ = norms.pop(0)
    x = pol.kept[0][1]
    assert same(gx, x) and gy is None and gz is None and same(gdx_out, dx) and same(gdn, dn)
    want = blocks.norm_backward(host(x), w_pre=host(pol.blocks[0].w_pre), dx_out=host(dx), dn=host(dn))
    near(dx_in, want["dx"], tol)
    near(grads["0.w_pre"], want["dw_pre"], 1e-4)
    assert matrix(pol.embed, pol.rows, dx_in, grads["embed"]) is None
    assert np.mean(tight) > 0.5         # (a sum over steps may come out near nothing)


def test_the_last_norms_weights_against_differences():
    """Of sum(n dn), n what the head gets and dn its gradient: the weights around the last block pass no
    4-bit product on the way there (behind the head's, whose rounding moves in steps, there is nothing to
    take differences of).  The differences' own error: eps^2 of third derivatives, 1e-4 of values of
    about 1; sums of M D rounded terms 1e-6."""
    pol, obs, done, dmu, dls = setup(torch.float32, 1)
    pol.forward(obs, done)
    grads = {k: v.clone() for k, v in pol.gradients(dmu, dls).items()}
    M = done.numel()
    dn = torch.empty(M, pol.D, device="cuda")
    tp.mx4_linear(dmu.view(M, -1), pol.head.wt4, dn)
    g, eps = torch.Generator("cuda").manual_seed(7), 1e-2
    for name in ("w_out", "0.w_post", "0.scale"):
        p = pol.parameters()[name]
        keep, d = p.clone(), torch.randn(p.shape, generator=g, device="cuda")
        sums = []
        for sign in (1, -1):
            p.copy_(keep + sign * eps * d)
            pol.forward(obs, done)
            sums.append((pol.last.double() * dn.double()).sum().item())
        p.copy_(keep)
        want, got = (sums[0] - sums[1]) / (2 * eps), (grads[name].double() * d.double()).sum().item()
        size = (grads[name].double() * d.double()).abs().sum().item()
        assert abs(got - want) <= 1e-3 * size, (name, got, want, size)
        assert abs(got) > 0.01 * size, (name, got, size)
