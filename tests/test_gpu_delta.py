"""Gated delta rule on the GPU against the 64-bit oracle.

Tolerances, relative to max(|value|, RMS of the array, size of the terms).  Values, states and their
gradients come in as N(0, 1), so every output is a sum of terms of about 1 (over its row's length for
q and k, whose gradients are divided by it); where few such terms cancel (one channel: 0.8 - 0.8 +
1e-4) the rounding is that of the terms, not of the value or, in an array of one, of its RMS.  A piece of up to 16 steps adds roundings of
2^-24 in sums of up to 128 + 16 products of its state and its writes: about sqrt(144) = 12 of them,
7e-7.  A head with a memory of M <= 2,000 steps gathers sqrt(M / 16) = 11 pieces' worth, 8e-6; the
gradients read states and run through as many pieces again: 2e-5 for all.  Outputs in bf16 add one
rounding of 2^-8.  r's gradient is a sum of dot products of up to 32 steps, which cancel: 2e-6 (32
roundings of 2^-24) of the lengths of the vectors in it; lambda's the same over all steps.
"""

import numpy as np
import pytest
import torch

from gpu_common import say
from oracle import delta
from paper_2111_05188_amd import tp
from test_gpu_recur import dev, host

pytestmark = pytest.mark.gpu

TOL = {torch.float32: 2e-5, torch.bfloat16: 2e-5 + 2.0 ** -8}
BOTH = [torch.float32, torch.bfloat16]


def close(name, got, want, tol, terms=1.0):
    got, want = np.asarray(got, np.float64), np.asarray(want, np.float64)
    fin = np.isfinite(want)
    assert np.array_equal(fin, np.isfinite(got)), name
    rms = np.sqrt(np.mean(want[fin] ** 2)) if fin.any() else 0.0
    size = np.maximum(np.maximum(np.abs(want), rms), np.broadcast_to(terms, want.shape))
    # (bf16: the rounding is the value's, the rest the terms')
    half = 2.0 ** -8 if tol > 2.0 ** -8 else 0.0
    bound = (tol - half) * size + half * np.maximum(np.abs(want), rms)
    bad = np.abs(got[fin] - want[fin]) > bound[fin]
    assert not bad.any(), (name, bad.sum(), np.abs(got[fin] - want[fin]).max(), rms)


def lambdas(g, H):
    a = 1.0 - 10.0 ** -(1.0 + 2.3 * g.random(H))
    return np.log(np.expm1(-np.log(a) / 4.0)).astype(np.float32)


class Case:
    """Inputs as views of one [T][B][N] array (or of one [B][T][N]) with `off` elements before
    them, and what they hold in 64 bits."""

    def __init__(self, T, B, H, dk, dv, dtype, done=0.0, ragged=False, seed=0, order="time", off=0,
                 junk=False, gate=1.0):
        g = np.random.default_rng(seed)
        self.T, self.B, self.H, self.dk, self.dv, self.dtype = T, B, H, dk, dv, dtype
        self.order, self.off = order, off
        self.done = (g.random((T, B)) < done).astype(np.uint8) if done else None
        self.lens = g.integers(0, T + 1, B).astype(np.int32) if ragged else None
        if ragged and B > 1:
            self.lens[0], self.lens[-1] = 0, T
        n = H * (2 * dk + dv + 2)
        rows = g.normal(size=(T, B, n)).astype(np.float32)
        rows[..., -2 * H:] *= gate
        dy = g.normal(size=(T, B, H * dv)).astype(np.float32)
        if junk:                        # what lies past a sequence's end does not matter
            for b in range(B):
                for v in (rows, dy):
                    v[self.lens[b]:, b] = np.resize([np.nan, np.inf, -np.inf], v.shape[2])
        self.rows, self.dy_rows = self.place(rows), self.place(dy)
        self.lam = lambdas(g, H)
        self.h0 = g.normal(size=(B, H, dk, dv)).astype(np.float32)
        self.dh = g.normal(size=(B, H, dk, dv)).astype(np.float32)
        self.out = self.place(np.zeros_like(rows)).fill_(7.0)
        self.setup()

    def setup(self):
        self.dc = tp.DeltaT(dev(self.lam), self.T, self.B, self.dk, self.dv, self.dtype,
                            done=None if self.done is None else dev(self.done),
                            lens=None if self.lens is None else dev(self.lens))
        self.work = self.dc.workspace()

    def place(self, v):
        t = dev(v, self.dtype)
        if self.order != "time":
            t = t.transpose(0, 1)
        a = torch.full((t.shape[0], t.shape[1], t.shape[2] + self.off), 3.0, dtype=self.dtype,
                       device="cuda")
        a[..., self.off:] = t
        a = a[..., self.off:]
        return a if self.order == "time" else a.transpose(0, 1)

    def parts(self, p):
        H, dk, dv = self.H, self.dk, self.dv
        at = np.cumsum([0, H * dk, H * dk, H * dv, H, H])
        q, k, v, r, b = (p[..., i:j] for i, j in zip(at, at[1:]))
        return (q.unflatten(-1, (H, dk)), k.unflatten(-1, (H, dk)), v.unflatten(-1, (H, dv)), r, b)

    @property
    def dy(self):
        return self.dy_rows.unflatten(-1, (self.H, self.dv))

    def exact_inputs(self):
        v = [np.nan_to_num(host(x), nan=1.0, posinf=1.0, neginf=1.0) for x in self.parts(self.rows)]
        return dict(zip("qkvrb", v), lam=self.lam.astype(np.float64),
                    h0=self.h0.astype(np.float64), done=self.done, lens=self.lens)

    def forward(self, saved=None, h0=True, y=True):
        y = torch.full((self.T, self.B, self.H, self.dv), 7.0, dtype=self.dtype,
                       device="cuda") if y else None
        last = torch.full((self.B, self.H, self.dk, self.dv), 7.0, device="cuda")
        tp.delta_forward(self.dc, *self.parts(self.rows), y, self.work,
                         h0=dev(self.h0) if h0 else None, h_last=last, saved=saved)
        return y, last

    def backward(self, saved):
        dlam = torch.full((self.H,), 7.0, device="cuda")
        dh0 = torch.full((self.B, self.H, self.dk, self.dv), 7.0, device="cuda")
        tp.delta_backward(self.dc, *self.parts(self.rows), saved, self.dy, *self.parts(self.out),
                          dlam, self.work, dh_last=dev(self.dh), dh0=dh0)
        return dlam, dh0

    def check(self):
        saved = self.dc.saved()
        y, last = self.forward(saved)
        dlam, dh0 = self.backward(saved)
        torch.cuda.synchronize()
        tol = TOL[self.dtype]
        e = self.exact_inputs()
        wy, wl = delta.forward(**e)
        close("y", host(y), wy, tol)
        close("h_last", host(last), wl, 2e-5)
        dy = np.nan_to_num(host(self.dy), nan=1.0, posinf=1.0, neginf=1.0)
        want = delta.backward(**e, dy=dy, dh_last=self.dh.astype(np.float64))
        got = dict(zip(("dq", "dk", "dv", "dr", "db"), self.parts(self.out)))
        for name in ("dq", "dk", "dv", "db"):
            close(name, host(got[name]), want[name], tol, want.get(name + "_size", 1.0))
        close("dh0", host(dh0), want["dh0"], 2e-5)
        rounding = 2.0 ** -8 if self.dtype == torch.bfloat16 else 2.0 ** -22
        err = np.abs(host(got["dr"]) - want["dr"])
        over = err - (rounding * np.abs(want["dr"]) + 2e-6 * want["dr_mass"] + 1e-30)
        at = np.unravel_index(over.argmax(), over.shape)
        assert over.max() <= 0, ("dr", at, err[at], want["dr"][at], want["dr_mass"][at])
        err = np.abs(host(dlam) - want["dlam"])
        fine = (err <= 2e-6 * want["dlam_mass"] + 1e-30).all()
        assert fine, ("dlam", err, want["dlam_mass"])


# one step; pieces of 16 and groups of 32 and their neighbours; several groups; one channel, odd
# ones, narrow keys with wide values and the other way round, whole heads of each width
SHAPES = [(1, 1, 1, 1, 1), (1, 3, 2, 64, 64), (2, 2, 1, 5, 3), (15, 2, 2, 32, 32), (16, 1, 3, 33, 31),
          (17, 2, 1, 64, 64), (31, 2, 2, 48, 64), (32, 1, 2, 128, 128), (33, 1, 3, 100, 48),
          (65, 2, 1, 128, 16), (100, 2, 1, 17, 127), (97, 7, 3, 32, 20), (200, 2, 2, 64, 64),
          (130, 1, 1, 128, 128)]


@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("done,ragged", [(0.0, False), (0.06, True)])
def test_sequences_and_gradients(shape, dtype, done, ragged):
    say(f"[delta] {shape} {dtype} done={done} ragged={ragged}")
    Case(*shape, dtype, done, ragged, seed=sum(shape)).check()


@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("shape", [(20, 300, 8, 64, 64), (40, 1100, 1, 32, 32)])
def test_many_sequences(shape, dtype):
    say(f"[delta] many {shape} {dtype}")
    Case(*shape, dtype, 0.05, True, seed=3).check()


@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("shape", [(700, 1, 2, 64, 64), (900, 3, 1, 32, 48), (500, 1, 1, 128, 128)])
@pytest.mark.parametrize("done,ragged", [(0.0, False), (0.004, True)])
def test_few_long_sequences(shape, dtype, done, ragged):
    say(f"[delta] long {shape} {dtype}")
    Case(*shape, dtype, done, ragged, seed=5).check()


@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("shape", [(3205, 1, 1, 32, 32), (4400, 2, 2, 16, 64), (3700, 1, 1, 128, 96)])
@pytest.mark.parametrize("done,ragged", [(0.0, False), (0.001, True)])
def test_very_long_sequences(shape, dtype, done, ragged):
    """So many segments that their states are joined over blocks of them."""
    say(f"[delta] very long {shape} {dtype}")
    Case(*shape, dtype, done, ragged, seed=6).check()


@pytest.mark.parametrize("dtype", BOTH)
def test_a_bad_number_far_before_an_episodes_end(dtype):
    """It stays in its episode, over segments and blocks of them; the states may be one buffer."""
    T = 3800
    c = Case(T, 1, 2, 32, 32, dtype, seed=15)
    c.done = np.zeros((T, 1), np.uint8)
    c.done[3000] = 1
    c.setup()
    y0, h0 = c.forward()
    c.parts(c.rows)[2][500, 0, 1, 3] = float("nan")
    y, state = torch.full_like(y0, 7.0), dev(c.h0)
    tp.delta_forward(c.dc, *c.parts(c.rows), y, c.work, h0=state, h_last=state)
    torch.cuda.synchronize()
    y0, y, h0, h = host(y0), host(y), host(h0), host(state)
    same = np.ones(y.shape, bool)
    same[500:3001, 0, 1] = False
    close("y", y[same], y0[same], 2 * TOL[dtype])
    close("h_last", h, h0, 4e-5)
    assert np.isnan(y[500:3001, 0, 1, 3]).all() and np.isfinite(y[500:3001, 0, 1, :3]).all()


@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("T", [90, 900])
def test_bad_states_stay_in_their_episodes(T, dtype):
    """A NaN in the first states reaches the first episode, one in the last states' gradient the
    last one: not the others', whose steps share groups and pieces of them."""
    c = Case(T, 1, 2, 64, 48, dtype, seed=16)
    ends = [T - 50, T - 30, T - 27, T - 3]
    c.done = np.zeros((T, 1), np.uint8)
    c.done[ends] = 1
    c.setup()

    def run():
        saved = c.dc.saved()
        y, last = c.forward(saved)
        c.out.fill_(7.0)
        _, dh0 = c.backward(saved)
        torch.cuda.synchronize()
        return [host(x) for x in (y, *c.parts(c.out), last, dh0)]

    fine = run()
    assert all(np.isfinite(x).all() for x in fine)
    tol = 2 * TOL[dtype]
    c.h0[0, 1, 5, 3], keep = np.nan, c.h0[0, 1, 5, 3]
    got = run()
    for name, x, y in zip(("y", "dq", "dk", "dv", "dr", "db"), got, fine):
        close(name + " after", x[ends[0] + 1:], y[ends[0] + 1:], tol)
        close(name + " of the other head", x[:, :, 0], y[:, :, 0], tol)
    close("h_last", got[6], fine[6], tol)
    assert np.isnan(got[0][:ends[0] + 1, 0, 1, 3]).all()
    c.h0[0, 1, 5, 3] = keep
    c.dh[0, 1, 5, 3] = np.nan
    got = run()
    for name, x, y in zip(("y", "dq", "dk", "dv", "dr", "db"), got, fine):
        close(name + " before", x[:ends[-1] + 1], y[:ends[-1] + 1], tol)
        close(name + " of the other head", x[:, :, 0], y[:, :, 0], tol)
    close("dh0", got[7], fine[7], tol)
    assert np.isnan(got[2][ends[-1] + 1:, 0, 1]).any()


@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("done", [1.0, 0.5])
@pytest.mark.parametrize("T", [1, 40, 75])
def test_episodes_of_one_and_few_steps(T, done, dtype):
    Case(T, 3, 2, 64, 32, dtype, done, seed=T).check()


@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("order,off", [("time", 3), ("batch", 0), ("batch", 5), ("time", 8)])
def test_layouts(order, off, dtype):
    """Parts of wider rows, sequence after sequence, rows that start off 16 bytes."""
    for d in ((64, 64), (40, 24)):
        Case(37, 3, 2, *d, dtype, 0.05, True, seed=off, order=order, off=off).check()


@pytest.mark.parametrize("dtype", BOTH)
def test_what_lies_past_a_sequence_does_not_matter(dtype):
    Case(70, 5, 2, 64, 64, dtype, 0.05, True, seed=9, junk=True).check()


@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("gate", [0.0, 8.0, 30.0])
def test_gates_of_any_strength(dtype, gate):
    """Gates at one half, and pre-activations up to 100: closed and open to the last digit."""
    Case(80, 2, 2, 64, 64, dtype, 0.0, False, seed=2, gate=gate).check()


@pytest.mark.parametrize("dtype", BOTH)
def test_the_same_key_again_and_again(dtype):
    """The triangle of a piece at its worst: all keys alike, every write at nearly full strength,
    no decay."""
    c = Case(64, 1, 2, 64, 64, dtype, seed=4)
    q, k, v, r, b = c.parts(c.rows)
    k.copy_(k[:1].expand_as(k).clone())
    b.fill_(6.0)
    r.fill_(-20.0)
    c.check()


@pytest.mark.parametrize("dtype", BOTH)
def test_zero_queries_and_keys(dtype):
    c = Case(40, 2, 1, 32, 32, dtype, seed=6)
    q, k, *_ = c.parts(c.rows)
    q[3:9], k[5:20] = 0.0, 0.0
    saved = c.dc.saved()
    y, last = c.forward(saved)
    c.backward(saved)
    wy, wl = delta.forward(**c.exact_inputs())
    close("y", host(y), wy, TOL[dtype])
    close("h_last", host(last), wl, 2e-5)
    assert (host(y)[3:9] == 0).all() and np.isfinite(host(c.out)).all()


@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("what", range(5))
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_a_bad_number_reaches_nothing_before_it(what, bad, dtype):
    """Nor other sequences, other heads, or what follows its episode."""
    c = Case(90, 2, 2, 64, 64, dtype, seed=8)
    c.done = np.zeros((90, 2), np.uint8)
    c.done[60] = 1
    c.setup()
    y0, h0 = c.forward()
    x = c.parts(c.rows)[what]
    x[41, 0, 1] = bad
    y, h = c.forward()
    torch.cuda.synchronize()
    y0, y, h0, h = host(y0), host(y), host(h0), host(h)
    same = np.ones(y.shape, bool)
    same[41:61, 0, 1] = False
    # (the steps before it are pieces of their own then: other roundings, not other values)
    close("y", y[same], y0[same], 2 * TOL[dtype])
    close("h_last", h, h0, 4e-5)
    if not (what == 4 or (what == 3 and np.isinf(bad))):    # (a gate at infinity is an open one)
        assert not np.isfinite(y[41:61, 0, 1]).all()


@pytest.mark.parametrize("dtype", BOTH)
def test_no_first_states_no_outputs(dtype):
    c = Case(50, 2, 2, 64, 64, dtype, seed=11)
    y, last = c.forward(h0=False)
    e = c.exact_inputs()
    e["h0"] = None
    wy, wl = delta.forward(**e)
    close("y", host(y), wy, TOL[dtype])
    close("h_last", host(last), wl, 2e-5)
    saved, only = c.dc.saved(), c.dc.saved()
    c.forward(saved)
    _, last2 = c.forward(only, y=False)
    assert torch.equal(saved, only)
    # dh_last and dh0 left out: zeros, not asked for
    dlam = torch.empty(2, device="cuda")
    tp.delta_backward(c.dc, *c.parts(c.rows), saved, c.dy, *c.parts(c.out), dlam, c.work)
    want = delta.backward(**c.exact_inputs(), dy=host(c.dy))
    close("dq", host(c.parts(c.out)[0]), want["dq"], TOL[dtype])


@pytest.mark.parametrize("dtype", BOTH)
def test_states_in_place_and_a_sequence_in_parts(dtype):
    c = Case(100, 3, 2, 64, 48, dtype, 0.03, seed=12)
    y, last = c.forward()
    state, ys = dev(c.h0), []
    for t0, t1 in ((0, 1), (1, 40), (40, 100)):
        dc = tp.DeltaT(dev(c.lam), t1 - t0, 3, 64, 48, dtype, done=dev(c.done[t0:t1]))
        part = torch.empty(t1 - t0, 3, 2, 48, dtype=dtype, device="cuda")
        tp.delta_forward(dc, *(x[t0:t1] for x in c.parts(c.rows)), part, dc.workspace(), h0=state,
                         h_last=state)
        ys.append(part)
    close("y", host(torch.cat(ys)), host(y), 2 * TOL[dtype])
    close("h_last", host(state), host(last), 4e-5)


@pytest.mark.parametrize("dtype", BOTH)
def test_gradient_states_in_place(dtype):
    c = Case(70, 3, 2, 32, 32, dtype, seed=13)
    saved = c.dc.saved()
    c.forward(saved)
    _, want = c.backward(saved)
    both, dlam = dev(c.dh), torch.empty(2, device="cuda")
    tp.delta_backward(c.dc, *c.parts(c.rows), saved, c.dy, *c.parts(c.out), dlam, c.work,
                      dh_last=both, dh0=both)
    assert torch.equal(both, want)


@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("shape", [(1, 1, 1, 1), (3, 2, 64, 64), (5, 3, 33, 127), (2, 1, 128, 128),
                                   (700, 4, 32, 32), (2, 2, 16, 100)])
@pytest.mark.parametrize("off", [0, 3])
def test_steps(shape, dtype, off):
    """A step is a sequence of one, in place too, with the states' ends."""
    B, H, dk, dv = shape
    c = Case(1, B, H, dk, dv, dtype, 0.3, seed=B, off=off)
    y, last = c.forward()
    parts = [x[0] for x in c.parts(c.rows)]
    h, lam, done = dev(c.h0), dev(c.lam), dev(c.done[0])
    out, ys = torch.full_like(h, 7.0), torch.full((B, H, dv), 7.0, dtype=dtype, device="cuda")
    tp.delta_step(*parts, lam, h, out, ys, done=done)
    wy, wl = delta.forward(**c.exact_inputs())
    close("y", host(ys), wy[0], TOL[dtype])
    close("h", host(out), wl, 2e-5)
    close("y of a sequence", host(y)[0], wy[0], TOL[dtype])
    tp.delta_step(*parts, lam, h, h, None, done=done)
    assert torch.equal(h, out)
    # states that start off 16 bytes
    a = torch.empty(h.numel() + 1, device="cuda")[1:].view(h.shape)
    a.copy_(dev(c.h0))
    tp.delta_step(*parts, lam, a, a, None, done=done)
    assert torch.equal(a, out)


def test_the_same_bits_every_time():
    c = Case(100, 4, 2, 64, 64, torch.bfloat16, 0.05, True, seed=14)
    saved = c.dc.saved()
    y, last = c.forward(saved)
    dlam, dh0 = c.backward(saved)
    out = c.out.clone()
    c.work.fill_(255)
    again = c.dc.saved().fill_(float("nan"))
    y2, last2 = c.forward(again)
    dlam2, dh02 = c.backward(again)
    for a, b in ((y, y2), (last, last2), (dlam, dlam2), (dh0, dh02), (out, c.out)):
        assert torch.equal(a, b)


def test_rows_that_are_not_the_operators_stay():
    """Around the parts of the rows, and past the states."""
    c = Case(40, 3, 2, 40, 24, torch.bfloat16, 0.0, True, seed=15, off=7)
    wide = c.out._base if c.out._base is not None else c.out
    before = wide[..., :7].clone()
    saved = torch.full((c.dc.saved_count + 64,), 5.0, device="cuda")
    c.forward(saved)
    c.backward(saved)
    assert torch.equal(wide[..., :7], before) and (saved[c.dc.saved_count:] == 5.0).all()


@pytest.mark.parametrize("dtype", BOTH)
def test_graph_replays(dtype):
    c = Case(60, 4, 2, 64, 64, dtype, 0.05, True, seed=16)
    saved, state = c.dc.saved(), dev(c.h0)
    y = torch.empty(60, 4, 2, 64, dtype=dtype, device="cuda")
    dlam, dh0, dh = torch.empty(2, device="cuda"), torch.empty_like(state), dev(c.dh)
    parts, out = c.parts(c.rows), c.parts(c.out)
    step_y = torch.empty(4, 2, 64, dtype=dtype, device="cuda")

    def run():
        tp.delta_forward(c.dc, *parts, y, c.work, h0=state, h_last=state, saved=saved)
        tp.delta_backward(c.dc, *parts, saved, c.dy, *out, dlam, c.work, dh_last=dh, dh0=dh0)
        tp.delta_step(*(x[0] for x in parts), c.dc.lam, state, state, step_y)

    def results():
        return [x.clone() for x in (y, state, dlam, dh0, c.out, step_y)]

    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    want, got = [], []
    state.copy_(dev(c.h0))
    for _ in range(4):
        run()
        want.append(results())
    state.copy_(dev(c.h0))
    for _ in range(4):
        graph.replay()
        got.append(results())
        torch.cuda.synchronize()
        torch.ones(1000, device="cuda").sum().item()
    for a, b in zip(want, got):
        assert all(torch.equal(x, z) for x, z in zip(a, b))


def test_another_stream():
    c = Case(60, 4, 2, 64, 64, torch.float32, seed=17)
    want, last = c.forward()
    s = torch.cuda.Stream()
    y, h = torch.empty_like(want), torch.empty_like(last)
    h0 = dev(c.h0)
    torch.cuda.synchronize()
    tp.delta_forward(c.dc, *c.parts(c.rows), y, c.work, h0=h0, h_last=h, stream=s)
    s.synchronize()
    assert torch.equal(y, want) and torch.equal(h, last)


def test_offsets_past_32_bits():
    """Rows more than 2^31 elements apart: two steps at the far ends of a large array."""
    H, d = 1, 64
    n = 3 * d + 2
    far = (1 << 31) + 8
    base = torch.zeros(far + n, dtype=torch.bfloat16, device="cuda")
    c = Case(2, 1, H, d, d, torch.bfloat16, seed=18)
    rows = torch.as_strided(base, (2, 1, n), (far, n, 1))
    rows.copy_(c.rows)
    y = torch.empty(2, 1, H, d, dtype=torch.bfloat16, device="cuda")
    want, _ = c.forward()
    tp.delta_forward(c.dc, *c.parts(rows), y, c.work, h0=dev(c.h0))
    assert torch.equal(y, want)


def test_refusals_on_the_gpu():
    c = Case(4, 2, 1, 8, 8, torch.float32)
    with pytest.raises(tp.TPError):
        tp.delta_forward(c.dc, *c.parts(c.rows), c.dy, c.work[:8])
    with pytest.raises(tp.TPError):
        tp.delta_forward(c.dc, *c.parts(c.rows), None, c.work)


@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("what", range(6))
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("T", [90, 800])
def test_a_bad_numbers_gradients_stay_in_its_episode(what, bad, T, dtype):
    """In an input or (5) dy: the gradients of other episodes, heads and sequences, and the first
    states' of the others, are as without it."""
    c = Case(T, 2, 2, 64, 64, dtype, seed=17)
    first, last = T - 70, T - 30
    c.done = np.zeros((T, 2), np.uint8)
    c.done[[first, last], 0] = 1
    c.setup()

    def run():
        saved = c.dc.saved()
        c.forward(saved)
        c.out.fill_(7.0)
        dlam, dh0 = c.backward(saved)
        torch.cuda.synchronize()
        return [host(x) for x in (*c.parts(c.out), dh0, dlam)]

    fine = run()
    x = (*c.parts(c.rows), c.dy)[what]
    x[T - 49, 0, 1] = bad
    got = run()
    for name, a, b in zip(("dq", "dk", "dv", "dr", "db"), got, fine):
        same = np.ones(a.shape, bool)
        same[first + 1:last + 1, 0, 1] = False
        close(name, a[same], b[same], 2 * TOL[dtype])
    close("dh0", got[5], fine[5], 4e-5)
    close("dlam", got[6][:1], fine[6][:1], 4e-5)
    if what in (0, 1, 2, 5):
        assert not np.isfinite(got[1][first + 1:last + 1, 0, 1]).all()


def test_two_calls_at_once_and_a_graph_of_many_segments():
    cases = [Case(2000, 1, 2, 64, 64, torch.bfloat16, 0.002, seed=18),
             Case(3600, 1, 1, 32, 64, torch.float32, 0.001, seed=19)]

    def run(c, o):
        tp.delta_forward(c.dc, *c.parts(c.rows), o["y"], c.work, h0=o["h0"], h_last=o["last"],
                         saved=o["saved"])
        tp.delta_backward(c.dc, *c.parts(c.rows), o["saved"], c.dy, *c.parts(c.out), o["dlam"], c.work,
                          dh_last=o["dh"], dh0=o["dh0"])

    outs, want = [], []
    for c in cases:
        h0 = dev(c.h0)
        o = dict(y=torch.empty(c.T, c.B, c.H, c.dv, dtype=c.dtype, device="cuda"), h0=h0,
                 last=torch.empty_like(h0), saved=c.dc.saved(), dh=dev(c.dh), dh0=torch.empty_like(h0),
                 dlam=torch.empty(c.H, device="cuda"))
        run(c, o)
        outs.append(o)
        want.append([o[k].clone() for k in ("y", "last", "dlam", "dh0")] + [c.out.clone()])
    torch.cuda.synchronize()

    def check(c, o, w):
        got = [o[k] for k in ("y", "last", "dlam", "dh0")] + [c.out]
        assert all(torch.equal(a, b) for a, b in zip(got, w))

    streams = [torch.cuda.Stream() for _ in cases]
    for _ in range(3):
        for c, o, s in zip(cases, outs, streams):
            c.out.zero_()
            o["y"].zero_()
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                run(c, o)
        torch.cuda.synchronize()
        for c, o, w in zip(cases, outs, want):
            check(c, o, w)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for c, o in zip(cases, outs):
            run(c, o)
    for _ in range(3):
        for c, o in zip(cases, outs):
            c.out.zero_()
            o["y"].zero_()
        graph.replay()
        torch.cuda.synchronize()
        for c, o, w in zip(cases, outs, want):
            check(c, o, w)
