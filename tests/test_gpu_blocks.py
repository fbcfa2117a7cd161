"""The norms around a block and the policy loss on the GPU against the 64-bit oracle.

Tolerances, relative to max(|value|, RMS of the array, size of the terms: where x and what is added
to it cancel, or a norm's gradient in a group of few channels, the rounding is that of the terms).
Norms: a row's sums of D <= 4,096 products
round by about sqrt(D) 2^-24 of their magnitude, 4e-6, halved by the root; the values around them add
ten roundings (the hardware's exponential and reciprocal among them): 8e-6.  Outputs in bf16 add one
rounding of 2^-8.  The weights' gradients are sums over rows: 8e-6 of the terms' sum of magnitudes.
The loss works in 64 bits: stats to 1e-12 of their magnitude, gradients one rounding of 2^-24 or 2^-8
(dlog_std, a sum that cancels, 2^-24 of itself and 1e-12 of its terms).
"""

import numpy as np
import pytest
import torch

from gpu_common import say
from oracle import blocks
from paper_2111_05188_amd import tp
from test_gpu_delta import close
from test_gpu_recur import dev, host

pytestmark = pytest.mark.gpu

BOTH = [torch.float32, torch.bfloat16]
TOL = {torch.float32: 8e-6, torch.bfloat16: 8e-6 + 2.0 ** -8}
ALL = ("x", "y", "z", "w_post", "scale", "w_pre")


class Norm:
    def __init__(self, M, D, groups, dtype, parts=ALL, seed=0, pad=0, off=0, size=1.0):
        g = np.random.default_rng(seed)
        self.M, self.D, self.groups, self.dtype, self.parts = M, D, groups, dtype, parts
        self.pad, self.off = pad, off
        t = {k: self.place(g.normal(size=(M, D)) * (size if k == "x" else 1.0))
             for k in ("x", "y", "z", "dx_out", "dn")}
        for k in ("w_post", "scale", "w_pre"):
            t[k] = dev(g.normal(size=D).astype(np.float32))
        if "w_pre" not in parts:
            t["dn"] = None
        self.t = {k: v for k, v in t.items() if k in parts or k in ("dx_out", "dn")}
        self.nc = tp.NormT(M, D, dtype, groups=groups,
                           **{k: self.t.get(k) for k in ("w_pre", "w_post", "scale")})

    def place(self, v):
        a = torch.full((self.M, self.D + self.pad + self.off), 3.0, dtype=self.dtype, device="cuda")
        a = a[:, self.off:self.off + self.D]
        a.copy_(torch.from_numpy(v))
        return a

    def new(self):
        return self.place(np.full((self.M, self.D), 7.0))

    def exact(self):
        return {k: host(self.t[k]) for k in self.parts}

    def forward(self):
        x_out, n = self.new(), self.new() if "w_pre" in self.parts else None
        tp.norm_forward(self.nc, self.t["x"], self.t.get("y"), self.t.get("z"), x_out, n)
        return x_out, n

    def backward(self, dx_out=True, dn=True):
        o = {"d" + k: self.new() if k in "xyz" else torch.full((self.D,), 7.0, device="cuda")
             for k in self.parts}
        tp.norm_backward(self.nc, self.t["x"], self.t.get("y"), self.t.get("z"),
                         self.t["dx_out"] if dx_out else None, self.t["dn"] if dn else None, o["dx"],
                         *(o.get("d" + k) for k in ("y", "z", "w_post", "scale", "w_pre")),
                         self.nc.workspace())
        return o

    def check(self):
        x_out, n = self.forward()
        got = self.backward()
        e, tol = self.exact(), TOL[self.dtype]
        X, wn, _ = blocks.norm_forward(**e, groups=self.groups)
        want = blocks.norm_backward(**e, groups=self.groups, dx_out=host(self.t["dx_out"]),
                                    dn=None if self.t["dn"] is None else host(self.t["dn"]))
        close("x_out", host(x_out), X, tol, want["x_size"])
        if n is not None:
            close("n", host(n), wn, tol, want["n_size"])
        for k, v in got.items():
            t = tol if k[1:] in "xyz" else 8e-6
            close(k, host(v), want[k], t, want[k + "_size"])


# one row, one channel; parts of a wave, a wave, several vectors a lane, a workgroup a row, with
# whole and odd vectors; groups of 2^k lanes, odd ones, groups of one channel
SIZES = [(1, 1, 1), (1, 64, 1), (5, 7, 7), (64, 64, 8), (33, 128, 1), (9, 256, 4), (70, 301, 1),
         (40, 100, 4), (3, 512, 8), (17, 768, 4), (6, 1001, 7), (5, 1024, 16), (4, 1500, 5),
         (3, 2048, 2), (2, 3001, 1), (2, 4096, 4), (3000, 96, 3), (9000, 33, 1), (5000, 256, 1)]


@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("size", SIZES)
def test_norms_and_gradients(size, dtype):
    say(f"[norm] {size} {dtype}")
    Norm(*size, dtype, seed=sum(size)).check()


@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("D,groups", [(129, 3), (191, 1), (193, 1), (255, 5), (257, 1), (319, 11), (321, 3),
                                      (383, 1), (385, 7), (511, 7), (513, 27), (1025, 5), (2049, 3)])
def test_rows_of_odd_lengths(D, groups, dtype):
    """On both sides of what a lane's registers hold."""
    Norm(13, D, groups, dtype, seed=D).check()


@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("parts", [("x", "w_pre"), ("x",), ("x", "y"), ("x", "y", "z"),
                                   ("x", "y", "w_post"), ("x", "y", "scale", "w_pre"),
                                   ("x", "y", "z", "w_post", "w_pre")])
@pytest.mark.parametrize("D", [64, 301])
def test_parts(parts, D, dtype):
    Norm(50, D, 1, dtype, parts, seed=1).check()


@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("pad,off", [(8, 0), (3, 0), (5, 3), (0, 8)])
def test_pitches(pad, off, dtype):
    """Parts of wider rows; what lies around them stays."""
    c = Norm(37, 128, 4, dtype, seed=2, pad=pad, off=off)
    c.check()
    x_out, _ = c.forward()
    base = x_out._base
    assert (base[:, :off] == 3.0).all() and (base[:, off + 128:] == 3.0).all()


@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("D", [128, 301, 2000])
def test_in_place(D, dtype):
    c = Norm(300, D, 1, dtype, seed=3)
    x_out, n = c.forward()
    want = c.backward()
    keep = c.t["dx_out"].clone()
    o = {k: torch.empty_like(want[k]) for k in want}
    tp.norm_backward(c.nc, c.t["x"], c.t["y"], c.t["z"], keep, c.t["dn"], keep, o["dy"], o["dz"],
                     o["dw_post"], o["dscale"], o["dw_pre"], c.nc.workspace())
    assert torch.equal(keep, want["dx"]) and torch.equal(o["dy"], want["dy"])
    assert all(torch.equal(o[k], want[k]) for k in ("dz", "dw_post", "dscale", "dw_pre"))
    x, n2 = c.t["x"].clone(), torch.empty_like(n)
    tp.norm_forward(c.nc, x, c.t["y"], c.t["z"], x, n2)
    assert torch.equal(x, x_out) and torch.equal(n2, n)


@pytest.mark.parametrize("dtype", BOTH)
def test_one_of_the_gradients_and_one_of_the_outputs(dtype):
    c = Norm(60, 256, 4, dtype, seed=4)
    e = c.exact()
    for a, b in ((True, False), (False, True), (False, False)):
        got = c.backward(a, b)
        want = blocks.norm_backward(**e, groups=4, dx_out=host(c.t["dx_out"]) if a else None,
                                    dn=host(c.t["dn"]) if b else None)
        for k in ("dx", "dy", "dz"):
            close(k, host(got[k]), want[k], TOL[dtype], want[k + "_size"])
        if not b:
            assert (host(got["dw_pre"]) == 0).all()
    X, n = c.forward()
    n2, X2 = torch.empty_like(n), torch.empty_like(X)
    tp.norm_forward(c.nc, c.t["x"], c.t["y"], c.t["z"], None, n2)
    tp.norm_forward(c.nc, c.t["x"], c.t["y"], c.t["z"], X2, None)
    assert torch.equal(n, n2) and torch.equal(X, X2)


@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("D,groups", [(64, 4), (768, 4), (301, 7)])
def test_bad_numbers_stay_in_their_rows_and_zeros_are_finite(D, groups, dtype):
    c = Norm(20, D, groups, dtype, seed=5)
    for k in ("x", "y"):
        c.t[k][3] = 0.0
    c.t["x"][7, 5], c.t["y"][9, 1], c.t["z"][11, 0] = float("nan"), float("inf"), float("nan")
    X, n = c.forward()
    o = c.backward()
    fine = np.ones(20, bool)
    fine[[7, 9, 11]] = False
    for t in (X, n, o["dx"], o["dy"], o["dz"]):
        assert np.isfinite(host(t)[fine]).all()
    assert (host(X)[3] == 0).all() and (host(n)[3] == 0).all()
    # a group with a NaN is one, the row's other groups add theirs to X as ever
    assert np.isfinite(host(X)[9, D // groups:]).all() and not np.isfinite(host(X)[9, 1])


@pytest.mark.parametrize("dtype", BOTH)
def test_norm_same_bits_graphs_and_streams(dtype):
    c = Norm(3000, 256, 4, dtype, seed=6)
    X, n = c.forward()
    o = c.backward()
    o2 = c.backward()
    assert all(torch.equal(o[k], o2[k]) for k in o)
    work, X2, n2 = c.nc.workspace(), torch.empty_like(X), torch.empty_like(n)
    g = {k: torch.empty_like(v) for k, v in o.items()}

    def run():
        tp.norm_forward(c.nc, c.t["x"], c.t["y"], c.t["z"], X2, n2)
        tp.norm_backward(c.nc, c.t["x"], c.t["y"], c.t["z"], c.t["dx_out"], c.t["dn"], g["dx"],
                         g["dy"], g["dz"], g["dw_post"], g["dscale"], g["dw_pre"], work)

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for i in range(3):
        for t in (X2, n2, *g.values()):
            t.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(X2, X) and torch.equal(n2, n) and all(torch.equal(g[k], o[k]) for k in o)
    s = torch.cuda.Stream()
    X2.fill_(7.0)
    torch.cuda.synchronize()
    tp.norm_forward(c.nc, c.t["x"], c.t["y"], c.t["z"], X2, n2, stream=s)
    s.synchronize()
    assert torch.equal(X2, X)


# --------------------------------------------------------------------------
# policy loss
# --------------------------------------------------------------------------

class Loss:
    def __init__(self, T, B, n, dtype, ragged=False, ref=True, seed=0, pad=0, kl=0.05, junk=False,
                 move=0.2):
        g = np.random.default_rng(seed)
        self.T, self.B, self.n, self.dtype, self.pad = T, B, n, dtype, pad
        ls_ref = (-1.0 + 0.2 * g.normal(size=n)).astype(np.float32)
        self.ls = (ls_ref + 0.05 * g.normal(size=n)).astype(np.float32)
        mu_ref = g.normal(size=(T, B, n)).astype(np.float32) * 0.5
        z = g.normal(size=(T, B, n))
        action = (mu_ref + np.exp(ls_ref) * z).astype(np.float32)
        logp = (-0.5 * z * z - ls_ref).sum(2) - 0.5 * n * blocks.LN_2PI
        mu = mu_ref + move / np.sqrt(n) * np.exp(ls_ref) * g.normal(size=(T, B, n))
        adv = g.normal(size=(T, B)).astype(np.float32)
        self.lens = g.integers(0, T + 1, B).astype(np.int32) if ragged else None
        if ragged and B > 1:
            self.lens[0], self.lens[-1] = 0, T
        if junk:
            past = np.arange(T)[:, None] >= self.lens
            for v in (mu, action, mu_ref, logp, adv):
                v[past] = np.nan
        self.ref = ref
        self.mu = self.place(mu)
        self.t = dict(action=dev(action), logp=dev(logp.astype(np.float32)), adv=dev(adv),
                      mu_ref=dev(mu_ref) if ref else None)
        self.kw = dict(clip=(0.2, 0.28), kl=kl if ref else 0.0, ent=0.02)
        self.ls_ref = ls_ref if ref else None
        self.setup()

    def setup(self):
        self.pc = tp.PolicyT(dev(self.ls), self.T, self.B, self.dtype, clip=self.kw["clip"],
                             kl_coef=self.kw["kl"], ent_coef=self.kw["ent"],
                             log_std_ref=None if self.ls_ref is None else dev(self.ls_ref),
                             lens=None if self.lens is None else dev(self.lens))
        self.work = self.pc.workspace()

    def place(self, v):
        a = torch.full((self.T, self.B, self.n + self.pad), 3.0, dtype=self.dtype, device="cuda")
        a[..., :self.n] = torch.from_numpy(np.asarray(v, np.float32)).to(self.dtype)
        return a[..., :self.n]

    def run(self):
        stats = torch.full((6,), 7.0, dtype=torch.float64, device="cuda")
        dmu, dls = self.place(np.full((self.T, self.B, self.n), 7.0)), torch.full((self.n,), 7.0, device="cuda")
        tp.policy_loss(self.pc, self.mu, self.t["action"], self.t["logp"], self.t["adv"], self.work,
                       stats, dmu, dls, mu_ref=self.t["mu_ref"])
        return stats, dmu, dls

    def exact(self):
        return dict(mu=host(self.mu), log_std=self.ls.astype(np.float64),
                    **{k: None if v is None else host(v) for k, v in self.t.items()},
                    log_std_ref=None if self.ls_ref is None else self.ls_ref.astype(np.float64),
                    lens=self.lens, **self.kw)

    def check(self):
        stats, dmu, dls = self.run()
        ws, wm, wl = blocks.policy_loss(**self.exact())
        size = np.abs(ws[1]) + self.kw["kl"] * np.abs(ws[2]) + 0.02 * np.abs(ws[3]) + 1.0
        fine = (np.abs(host(stats) - ws) <= 1e-12 * (np.abs(ws) + size) * self.n).all()
        assert fine, (host(stats), ws)
        half = 2.0 ** -8 if self.dtype == torch.bfloat16 else 2.0 ** -23
        got = host(dmu)
        fine = (np.abs(got - wm) <= half * np.abs(wm) + 1e-11 * np.abs(wm).max() + 1e-38).all()
        assert fine, np.abs(got - wm).max()
        fine = (np.abs(host(dls) - wl) <= 2.0 ** -23 * np.abs(wl) + 1e-11).all()
        assert fine, (host(dls), wl)
        if self.pad:
            assert (dmu._base[..., self.n:] == 3.0).all()


LOSSES = [(1, 1, 1), (1, 1, 100), (3, 5, 7), (4, 9, 8), (2, 3, 16), (5, 7, 30), (6, 50, 33), (3, 4, 64),
          (2, 9, 65), (4, 4, 128), (10, 30, 100), (7, 3, 126), (50, 200, 12), (30, 1000, 5)]


@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("shape", LOSSES)
@pytest.mark.parametrize("ragged,ref", [(False, True), (True, True), (True, False)])
def test_policy_loss(shape, dtype, ragged, ref):
    say(f"[loss] {shape} {dtype} {ragged} {ref}")
    Loss(*shape, dtype, ragged, ref, seed=sum(shape)).check()


@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("pad", [1, 2, 4, 8, 28])
def test_policy_loss_of_wider_rows(pad, dtype):
    for n in (5, 30, 100):
        Loss(4, 30, n, dtype, True, seed=pad, pad=pad).check()


@pytest.mark.parametrize("dtype", BOTH)
def test_rows_that_no_sequence_has(dtype):
    c = Loss(9, 12, 30, dtype, True, seed=1, junk=True)
    c.check()
    _, dmu, _ = c.run()
    past = torch.arange(9, device="cuda")[:, None] >= dev(c.lens)
    assert (dmu[past] == 0).all()
    c.lens[:] = 0                           # none at all
    c.setup()
    stats, dmu, dls = c.run()
    assert (dmu == 0).all() and (dls == -0.02).all() and np.isfinite(host(stats)).all()
    assert host(stats)[5] == 0
    c.lens[:] = [-3, 100] * 6               # clamped to 0..T
    c.setup()
    assert host(c.run()[0])[5] == 54


def test_the_learners_loss():
    """The same loss, entropy, clip fraction and gradient as the PPO learner's on its minibatch."""
    from oracle import ppo
    import workloads as W
    cfg = W.get_config("tiny")
    S, H1, H2, n = cfg.dims
    dims, B, rows = (S, H1, H2, n, H1, H2), 64, 256
    flat = W.make_flat_params(cfg)
    obs, action, adv, ret, which = W.make_learner_data(cfg, rows)
    p = ppo.unflatten(flat.astype(np.float64), dims)
    f = ppo.forward(p, obs[:, :S], bf16=False)
    logp = (ppo.log_prob(action, f["mu"], p["log_std"])
            - np.asarray(W.LOG_RATIO_OFFSETS)[which]).astype(np.float32)
    c = tp.ppo_cfg(dims, tp.TP_F32, B)
    P = tp.ppo_param_count(c)
    idx = np.random.default_rng(1).choice(rows, B, replace=False)
    prm, m, v = dev(flat.copy()), torch.zeros(P, device="cuda"), torch.zeros(P, device="cuda")
    grad, stats = torch.empty(P, device="cuda"), torch.empty(1, 4, dtype=torch.float64, device="cuda")
    tp.ppo_update(c, prm, m, v, 1, dev(obs), dev(action), dev(logp), dev(adv), dev(ret),
                  dev(idx[None].astype(np.int64)), tp.ppo_workspace(c), grad=grad, stats=stats)
    log_std = p["log_std"].astype(np.float32)
    pc = tp.PolicyT(dev(log_std), 1, B, torch.float32)
    mine = torch.empty(6, dtype=torch.float64, device="cuda")
    mu, dls = dev(f["mu"][idx].astype(np.float32)[None]), torch.empty(n, device="cuda")
    dmu = torch.empty_like(mu)
    tp.policy_loss(pc, mu, dev(action[idx][None]), dev(logp[idx][None]), dev(adv[idx][None]),
                   pc.workspace(), mine, dmu, dls)
    a, b = host(mine), host(stats)[0]
    # (the learner's own forward is fp32: 1e-5 of sums of some ten terms)
    assert abs(a[1] - b[0]) < 1e-4 and abs(a[3] - b[1]) < 1e-5 and abs(a[4] - b[3]) < 1e-6
    seg, _ = tp.flat_segments(dims)
    at = lambda k: host(grad[seg[k][0]:seg[k][0] + n])  # noqa: E731
    for got, want in ((host(dmu)[0].sum(0), at("b3")), (host(dls), at("log_std"))):
        assert np.linalg.norm(got - want) <= 1e-4 * np.linalg.norm(want)


@pytest.mark.parametrize("dtype", BOTH)
def test_a_bad_row_and_far_ratios(dtype):
    c = Loss(4, 6, 30, dtype, seed=2)
    c.t["logp"][1, 1] -= 2000.0             # a ratio past every number, a gain: clipped
    c.t["adv"][1, 1] = 1.0
    c.t["logp"][2, 2] += 2000.0             # and one of 0, a loss
    c.t["adv"][2, 2] = -1.0
    c.check()
    c.t["adv"][3, 3] = float("nan")
    stats, dmu, dls = c.run()
    assert np.isnan(host(stats)[1]) and not np.isnan(host(stats)[2])
    fine = torch.ones(4, 6, dtype=torch.bool, device="cuda")
    fine[3, 3] = False
    assert torch.isfinite(dmu[fine]).all()


@pytest.mark.parametrize("dtype", BOTH)
def test_loss_same_bits_graphs_and_streams(dtype):
    c = Loss(40, 300, 30, dtype, True, seed=3)
    a, b = c.run(), c.run()
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    outs = [torch.empty_like(x) for x in a]

    def run():
        tp.policy_loss(c.pc, c.mu, c.t["action"], c.t["logp"], c.t["adv"], c.work, *outs,
                       mu_ref=c.t["mu_ref"])

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for _ in range(3):
        for x in outs:
            x.fill_(7.0)
        c.work.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(a, outs))
    s = torch.cuda.Stream()
    for x in outs:
        x.fill_(7.0)
    torch.cuda.synchronize()
    tp.policy_loss(c.pc, c.mu, c.t["action"], c.t["logp"], c.t["adv"], c.work, *outs,
                   mu_ref=c.t["mu_ref"], stream=s)
    s.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(a, outs))


def test_policy_loss_of_many_sequences():
    """More sequences than a workgroup adds up lengths of; more rows than there are lanes."""
    for T, B, n in ((2, 8191, 3), (2, 8193, 3), (3, 30000, 1)):
        Loss(T, B, n, torch.float32, True, seed=B).check()
