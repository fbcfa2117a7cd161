"""Gated linear recurrence on the GPU against the 64-bit oracle.

Tolerances, relative to max(|value|, RMS of the array).  A step adds a few roundings of 2^-24 of
the state; a channel with a memory of M steps gathers about sqrt(M) of them.  With M <= 2,000 and
eight roundings (gates, their products, the sum) that is 8 * 6e-8 * 45 = 2e-5.  Outputs in bf16 add
one rounding of 2^-8.  lambda's gradient is a sum with cancellation: 2e-5 of the sum of magnitudes.
"""

import numpy as np
import pytest
import torch

from gpu_common import say
from oracle import recur
from paper_2111_05188_amd import tp

pytestmark = pytest.mark.gpu

TOL = {torch.float32: 2e-5, torch.bfloat16: 2e-5 + 2.0 ** -8}


def lambdas(g, D):
    a = 1.0 - 10.0 ** -(1.0 + 2.3 * g.random(D))
    return np.log(np.expm1(-np.log(a) / 4.0)).astype(np.float32)


def dev(x, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(x)).cuda()
    return t if dtype is None else t.to(dtype)


def host(t):
    return t.double().cpu().numpy()


def close(name, got, want, tol):
    got, want = np.asarray(got, np.float64), np.asarray(want, np.float64)
    fin = np.isfinite(want)
    assert np.array_equal(fin, np.isfinite(got)), name
    rms = np.sqrt(np.mean(want[fin] ** 2)) if fin.any() else 0.0
    err = np.abs(got[fin] - want[fin])
    bad = err > tol * np.maximum(np.abs(want[fin]), rms)
    assert not bad.any(), (name, bad.sum(), err.max(), rms)


class Case:
    """Inputs as views of one [T][B][3D] array (or of one [B][T][3D]), with what they hold in 64
    bits."""

    def __init__(self, T, B, D, dtype, done=0.0, ragged=False, seed=0, order="time", junk=False):
        g = np.random.default_rng(seed)
        self.T, self.B, self.D, self.dtype = T, B, D, dtype
        self.done = (g.random((T, B)) < done).astype(np.uint8) if done else None
        self.lens = g.integers(0, T + 1, B).astype(np.int32) if ragged else None
        if ragged and B > 1:
            self.lens[0], self.lens[-1] = 0, T
        gates = g.normal(size=(T, B, 3 * D)).astype(np.float32)
        dy = g.normal(size=(T, B, D)).astype(np.float32)
        if junk:                        # what lies past a sequence's end does not matter
            for b in range(B):
                for v, k in ((gates, 3 * D), (dy, D)):
                    v[self.lens[b]:, b] = np.resize([np.nan, np.inf, -np.inf], k)
        self.gates, self.dy = self.place(gates, order), self.place(dy, order)
        self.lam, self.h0 = lambdas(g, D), g.normal(size=(B, D)).astype(np.float32)
        self.dh = g.normal(size=(B, D)).astype(np.float32)
        self.out = self.place(np.zeros((T, B, 3 * D), np.float32), order).fill_(7.0)
        self.rc = tp.RecurT(dev(self.lam), T, B, dtype,
                            done=None if self.done is None else dev(self.done),
                            lens=None if self.lens is None else dev(self.lens))
        self.work = self.rc.workspace()

    def place(self, v, order):
        t = dev(v, self.dtype)
        return t if order == "time" else t.transpose(0, 1).contiguous().transpose(0, 1)

    def split(self, t):
        D = self.D
        return t[..., :D], t[..., D:2 * D], t[..., 2 * D:]

    def exact_inputs(self):
        x, r, i = (np.nan_to_num(host(v), nan=1.0, posinf=1.0, neginf=1.0)
                   for v in self.split(self.gates))
        return dict(x=x, r=r, i=i, lam=self.lam.astype(np.float64),
                    h0=self.h0.astype(np.float64), done=self.done, lens=self.lens)

    def forward(self, saved=None, h_last=True):
        y = torch.full((self.T, self.B, self.D), 7.0, dtype=self.dtype, device="cuda")
        last = torch.full((self.B, self.D), 7.0, device="cuda") if h_last else None
        tp.recur_forward(self.rc, *self.split(self.gates), y, self.work, h0=dev(self.h0),
                         h_last=last, saved=saved)
        return y, last

    def backward(self, saved):
        dlam = torch.full((self.D,), 7.0, device="cuda")
        dh0 = torch.full((self.B, self.D), 7.0, device="cuda")
        tp.recur_backward(self.rc, *self.split(self.gates), saved, self.dy, *self.split(self.out),
                          dlam, self.work, dh_last=dev(self.dh), dh0=dh0)
        return dlam, dh0

    def check(self):
        saved = self.rc.saved()
        y, last = self.forward(saved)
        dlam, dh0 = self.backward(saved)
        torch.cuda.synchronize()
        tol = TOL[self.dtype]
        e = self.exact_inputs()
        wy, wl = recur.forward(**e)
        close("y", host(y), wy, tol)
        close("h_last", host(last), wl, 2e-5)
        dy = np.nan_to_num(host(self.dy), nan=1.0, posinf=1.0, neginf=1.0)
        dx, dr, di, wlam, wh0, mass = recur.backward(**e, dy=dy,
                                                     dh_last=self.dh.astype(np.float64))
        for name, got, want in zip(("dx", "dr", "di"), self.split(self.out), (dx, dr, di)):
            close(name, host(got), want, tol)
        close("dh0", host(dh0), wh0, 2e-5)
        # (beta^2 below the smallest normal number, 1e-38, is not resolved: beta = 1e-19)
        assert (np.abs(host(dlam) - wlam) <= 2e-5 * mass + 1e-16).all(), "dlam"


BOTH = [torch.float32, torch.bfloat16]

# one step; chunks of 8 and their neighbours; tiles of 4 and 16 waves; several segments; one
# channel, odd ones, part of a wave, two lanes' worth
SHAPES = [(1, 1, 1), (1, 5, 64), (2, 3, 65), (7, 2, 70), (8, 2, 64), (9, 3, 33), (31, 2, 128),
          (33, 4, 130), (127, 2, 66), (129, 1, 5), (300, 3, 192), (1500, 1, 96), (2520, 2, 31)]


@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("done,ragged", [(0.0, False), (0.05, True)])
def test_sequences_and_gradients(shape, dtype, done, ragged):
    say(f"[recur] {shape} {dtype} done={done} ragged={ragged}")
    Case(*shape, dtype, done, ragged, seed=sum(shape)).check()


@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("shape", [(20, 1100, 64), (20, 2100, 66), (5, 4200, 128), (70, 600, 256)])
def test_many_sequences(shape, dtype):
    """Enough waves that a sequence gets one wave or four, two channels a lane; sampled sequences
    against the oracle, the rest against runs of their own."""
    say(f"[recur] many {shape} {dtype}")
    c = Case(*shape, dtype, 0.05, True, seed=3)
    saved = c.rc.saved()
    y, last = c.forward(saved)
    dlam, dh0 = c.backward(saved)
    torch.cuda.synchronize()
    pick = [0, 1, shape[1] // 2, shape[1] - 1]
    e = c.exact_inputs()
    e = {k: v if k == "lam" else v[pick] if k in ("h0", "lens") else v[:, pick]
         for k, v in e.items()}
    wy, wl = recur.forward(**e)
    tol = TOL[dtype]
    close("y", host(y)[:, pick], wy, tol)
    close("h_last", host(last)[pick], wl, 2e-5)
    dx, dr, di, _, wh0, _ = recur.backward(**e, dy=host(c.dy)[:, pick],
                                           dh_last=c.dh[pick].astype(np.float64))
    for name, got, want in zip(("dx", "dr", "di"), c.split(c.out), (dx, dr, di)):
        close(name, host(got)[:, pick], want, tol)
    close("dh0", host(dh0)[pick], wh0, 2e-5)
    # lambda's gradient by differentiating the same definition in 64 bits over all sequences
    g = c.gates.double()
    lam = dev(c.lam).double().requires_grad_()
    x, r, i = c.split(g)
    L = -8.0 * torch.nn.functional.softplus(lam) * torch.sigmoid(r)
    a, u = torch.exp(L), torch.sqrt(-torch.expm1(2.0 * L)) * torch.sigmoid(i) * x
    h, loss = dev(c.h0).double(), 0.0
    for t in range(shape[0]):
        live = (t < c.rc.lens)[:, None]
        new = a[t] * h + u[t]
        loss = loss + (torch.where(live, new, 0.0) * c.dy[t].double()).sum()
        h = torch.where(live, torch.where(c.rc.done[t][:, None] != 0, 0.0, new), h)
    loss = loss + (h * dev(c.dh).double()).sum()
    loss.backward()
    # w of a step is at most a few times |dy| memory: RMS over channels stands for the mass
    want = lam.grad
    assert ((dlam.double() - want).abs() <= 2e-5 * (want.abs() + want.square().mean().sqrt() *
                                                    shape[1] ** 0.5)).all()


@pytest.mark.parametrize("shape,dtype", [((64, 2100, 130), torch.float32),
                                         ((64, 2100, 256), torch.bfloat16)])
def test_more_than_the_last_level_cache_holds(shape, dtype):
    """Over 256 MB of two channels a lane and a wave a sequence: loads and stores past the caches."""
    test_many_sequences(shape, dtype)


@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("shape", [(33, 3, 66), (300, 2, 64), (20, 1100, 128)])
def test_nothing_past_a_sequences_end_matters(shape, dtype):
    """NaN and infinities in the steps past each length: outputs are those of clean inputs."""
    a, b = (Case(*shape, dtype, 0.05, True, seed=8, junk=j) for j in (True, False))
    res = []
    for c in (a, b):
        saved = c.rc.saved()
        res.append((*c.forward(saved), *c.backward(saved), c.out))
    torch.cuda.synchronize()
    for p, q in zip(*res):
        assert torch.equal(p, q)


@pytest.mark.parametrize("T", [12, 300, 2000])
def test_an_episodes_end_forgets_nan(T):
    """A NaN before an episode's end reaches neither the states after it nor, from behind, the
    gradients before it."""
    c = Case(T, 2, 64, torch.float32, seed=9)
    done = np.zeros((T, 2), np.uint8)
    cut = T // 2
    done[cut] = 1
    c.done = done
    c.rc = tp.RecurT(dev(c.lam), T, 2, torch.float32, done=dev(done))
    c.gates[cut - 2, 0, 3] = float("nan")       # x of channel 3
    saved = c.rc.saved()
    y, last = c.forward(saved)
    torch.cuda.synchronize()
    assert torch.isnan(y[cut - 2:cut + 1, 0, 3]).all()
    assert torch.isfinite(y[cut + 1:]).all() and torch.isfinite(last).all()
    c.gates[cut - 2, 0, 3] = 0.5
    c.dy[cut + 1, 1, 5] = float("nan")
    c.forward(saved)
    dlam, dh0 = c.backward(saved)
    torch.cuda.synchronize()
    dx = c.split(c.out)[0]
    assert torch.isnan(dx[cut + 1, 1, 5])
    assert torch.isfinite(dx[:cut + 1]).all() and torch.isfinite(dh0).all()
    assert torch.isnan(dlam[5]) and torch.isfinite(dlam[:5]).all()


# one wave a sequence; four waves; sixteen; segments over workgroups
SPLITS = [(40, 2100, 64), (40, 600, 64), (200, 2, 64), (6000, 1, 64)]


def decaying(T, B, D, dtype, seed, top):
    """Memories of a hundred bars to a fraction of one: products of decays underflow, over many
    steps or within a few."""
    c = Case(T, B, D, dtype, seed=seed)
    c.lam = np.linspace(-6.0, top, D).astype(np.float32)
    c.rc = tp.RecurT(dev(c.lam), T, B, dtype)
    return c


@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("T,B,D", SPLITS)
def test_nan_stays_to_the_end(T, B, D, dtype):
    """Without an episode's end a NaN state is NaN in every later step, however little of it a
    finite state would have left, and a NaN gradient in every earlier one."""
    say(f"[recur] nan stays {T, B, D} {dtype}")
    c = decaying(T, B, D, dtype, 21, 4.0)
    saved = c.rc.saved()
    c.gates[5, 0, :D] = float("nan")
    y, last = c.forward(saved)
    torch.cuda.synchronize()
    assert torch.isfinite(y[:5]).all() and torch.isnan(y[5:, 0]).all() and torch.isnan(last[0]).all()
    assert torch.isfinite(y[:, 1:]).all() and torch.isfinite(last[1:]).all()
    c.gates[5, 0, :D] = 0.5
    c.dy[T - 6, 0] = float("nan")
    c.forward(saved)
    dlam, dh0 = c.backward(saved)
    torch.cuda.synchronize()
    assert torch.isnan(c.out[:T - 5, 0]).all() and torch.isfinite(c.out[T - 5:]).all()
    assert torch.isnan(dh0[0]).all() and torch.isnan(dlam).all()
    assert torch.isfinite(c.out[:, 1:]).all() and torch.isfinite(dh0[1:]).all()


@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("T,B,D", SPLITS)
def test_infinity_stays(T, B, D, dtype):
    """An infinite state stays what it is under finite inputs, in steps past a sequence's end too,
    and so does an infinite gradient: a is never 0."""
    say(f"[recur] infinity stays {T, B, D} {dtype}")
    c = decaying(T, B, D, dtype, 22, 20.0)
    inf = float("inf")
    lens = np.full(B, T, np.int32)
    lens[-1] = T - 3 if B > 1 else T
    c.rc = tp.RecurT(c.rc.lam, T, B, dtype, lens=dev(lens))
    c.h0[0] = np.where(np.arange(D) % 2, inf, -inf)
    if B > 1:
        c.h0[-1] = inf
    want = dev(c.h0)
    saved = c.rc.saved()
    y, last = c.forward(saved)
    torch.cuda.synchronize()
    assert torch.equal(y[:, 0].float(), want[0].expand(T, D)) and torch.equal(last[0], want[0])
    if B > 1:
        assert (y[:T - 3, -1] == inf).all() and (y[T - 3:, -1] == 0).all() and (last[-1] == inf).all()
    assert torch.isfinite(y[:, 1:B - 1]).all()
    c.h0[:] = 0.5
    c.dh[0], c.dh[-1] = c.dh[-1], inf
    c.forward(saved)
    _, dh0 = c.backward(saved)
    torch.cuda.synchronize()
    assert (dh0[-1] == inf).all() and torch.isfinite(dh0[:B - 1]).all()
    dx = c.split(c.out)[0]
    assert (dx[:lens[-1], -1] == inf).all() and (dx[lens[-1]:, -1] == 0).all()


def test_an_infinite_state_steps_to_itself():
    for dtype in BOTH:
        c = decaying(1, 3, 256, dtype, 23, 20.0)
        h = torch.full((3, 256), float("-inf"), device="cuda")
        y = torch.empty(3, 256, dtype=dtype, device="cuda")
        tp.recur_step(*c.split(c.gates[0]), c.rc.lam, h, h, y)
        torch.cuda.synchronize()
        assert (h == float("-inf")).all() and (y == float("-inf")).all()


@pytest.mark.parametrize("dtype", BOTH)
def test_extreme_gates(dtype):
    """Gates shut and open to the last bit, lambda far out: results stay finite and right."""
    T, B = 40, 2
    lam = np.array([-200.0, -90.0, -20.0, 0.0, 20.0, 90.0, 1.0, -3.0], np.float32)
    c = Case(T, B, 8, dtype, seed=10)
    c.lam = lam
    c.rc = tp.RecurT(dev(lam), T, B, dtype)
    big = [-1e30, -200.0, -90.0, -30.0, 0.0, 30.0, 90.0, 200.0, 1e30]
    g = np.random.default_rng(11)
    gates = host(c.gates)
    pick = g.random(gates.shape) < 0.5
    pick[..., :8] = False                       # x stays ordinary
    gates[pick] = g.choice(big, pick.sum())
    c.gates = dev(gates.astype(np.float32), dtype)
    c.check()


@pytest.mark.parametrize("dtype", BOTH)
def test_strides_and_orders(dtype):
    """Sequence-major arrays, arrays whose parts are not aligned to two channels, broadcast inputs:
    the same numbers as from contiguous ones."""
    T, B, D = 37, 5, 66
    base = Case(T, B, D, dtype, 0.05, True, seed=12)
    saved = base.rc.saved()
    want = (*base.forward(saved), *base.backward(saved), base.out)
    other = Case(T, B, D, dtype, 0.05, True, seed=12, order="sequence")
    saved = other.rc.saved()
    got = (*other.forward(saved), *other.backward(saved), other.out)
    torch.cuda.synchronize()
    for p, q in zip(got, want):
        assert torch.equal(p, q)
    # parts at odd offsets
    wide = torch.zeros(T, B, 3 * D + 7, dtype=dtype, device="cuda")
    parts = [wide[..., k * (D + 1) + 1:k * (D + 1) + 1 + D] for k in range(3)]
    for p, v in zip(parts, base.split(base.gates)):
        p.copy_(v)
    y = torch.empty_like(want[0])
    last = torch.empty_like(want[1])
    tp.recur_forward(base.rc, *parts, y, base.work, h0=dev(base.h0), h_last=last)
    torch.cuda.synchronize()
    assert torch.equal(y, want[0]) and torch.equal(last, want[1])
    # one row of x for every sequence
    x = base.split(base.gates)[0][:, :1].expand(T, B, D)
    _, r, i = base.split(base.gates)
    tp.recur_forward(base.rc, x, r, i, y, base.work, h0=dev(base.h0))
    z = torch.empty_like(y)
    tp.recur_forward(base.rc, x.contiguous(), r, i, z, base.work, h0=dev(base.h0))
    torch.cuda.synchronize()
    assert torch.equal(y, z)


@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("B,D", [(1, 1), (3, 65), (64, 512), (1000, 66), (70000, 64)])
def test_step_continues_a_sequence(B, D, dtype):
    """Five single steps: each the oracle's step from the same state; in place and out of place."""
    c = Case(5, B, D, dtype, 0.2, seed=13)
    h = dev(c.h0)
    y = torch.empty(B, D, dtype=dtype, device="cuda")
    pick = np.unique([0, B // 2, B - 1])
    e = c.exact_inputs()
    for t in range(5):
        x, r, i = c.split(c.gates[t])
        before = host(h)
        out = torch.empty_like(h)
        tp.recur_step(x, r, i, c.rc.lam, h, out, y, done=c.rc.done[t].contiguous())
        tp.recur_step(x, r, i, c.rc.lam, h, h, None, done=c.rc.done[t].contiguous())
        torch.cuda.synchronize()
        assert torch.equal(h, out)
        wy, wh = recur.forward(*(e[k][t:t + 1, pick] for k in "xri"), e["lam"], before[pick],
                               c.done[t:t + 1, pick])
        close("y", host(y)[pick], wy[0], TOL[dtype])
        close("h", host(h)[pick], wh, 2e-5)


@pytest.mark.parametrize("dtype", BOTH)
@pytest.mark.parametrize("B,D", [(1000, 130), (300, 192), (32768, 516)])
def test_step_of_two_and_four_channels_a_lane(B, D, dtype):
    """The widths below 256, and steps of more bytes than the last-level cache holds."""
    test_step_continues_a_sequence(B, D, dtype)


def test_step_equals_the_sequence_kernel():
    c = Case(6, 40, 128, torch.float32, 0.2, seed=14)
    y, last = c.forward()
    h = dev(c.h0)
    for t in range(6):
        yt = torch.empty(40, 128, device="cuda")
        tp.recur_step(*c.split(c.gates[t]), c.rc.lam, h, h, yt, done=c.rc.done[t].contiguous())
        torch.cuda.synchronize()
        assert torch.equal(yt, y[t])
    assert torch.equal(h, last)


@pytest.mark.parametrize("T,B", [(40, 3), (300, 2), (20, 2100)])
def test_only_the_last_states(T, B):
    """y left out: the last states and what the gradients need are those of a call with it."""
    c = Case(T, B, 66, torch.bfloat16, 0.05, True, seed=20)
    saved, kept = c.rc.saved().zero_(), c.rc.saved().zero_()
    y, last = c.forward(saved)
    only = torch.empty_like(last)
    tp.recur_forward(c.rc, *c.split(c.gates), None, c.work, h0=dev(c.h0), h_last=only, saved=kept)
    torch.cuda.synchronize()
    assert torch.equal(only, last) and torch.equal(kept, saved)


def test_segments_continue():
    """A sequence in two calls, the state handed on, equals one call to rounding."""
    c = Case(200, 3, 64, torch.float32, 0.02, seed=15)
    y, last = c.forward()
    x, r, i = c.split(c.gates)
    h = dev(c.h0)
    for part in (slice(0, 90), slice(90, 200)):
        T = part.stop - part.start
        rc = tp.RecurT(c.rc.lam, T, 3, torch.float32, done=c.rc.done[part].contiguous())
        out, nxt = torch.empty(T, 3, 64, device="cuda"), torch.empty(3, 64, device="cuda")
        tp.recur_forward(rc, x[part], r[part], i[part], out, rc.workspace(), h0=h, h_last=nxt)
        torch.cuda.synchronize()
        close("y", host(out), host(y[part]), 2e-5)
        h = nxt
    close("h", host(h), host(last), 2e-5)


@pytest.mark.parametrize("T,B,D", SPLITS + [(24570, 1, 512), (2520, 16, 128)])
def test_states_in_place(T, B, D):
    """h_last in h0's buffer and dh0 in dh_last's: the bits of buffers of their own."""
    c = Case(T, B, D, torch.bfloat16, 0.01, seed=24)
    saved = c.rc.saved()
    y, last = c.forward(saved)
    _, dh0 = c.backward(saved)
    want = c.out.clone()
    for _ in range(3):
        h, g, z = dev(c.h0), dev(c.dh), torch.empty_like(y)
        c.out.fill_(7.0)
        dlam = torch.empty(D, device="cuda")
        tp.recur_forward(c.rc, *c.split(c.gates), z, c.work, h0=h, h_last=h, saved=saved)
        tp.recur_backward(c.rc, *c.split(c.gates), saved, c.dy, *c.split(c.out), dlam, c.work,
                          dh_last=g, dh0=g)
        torch.cuda.synchronize()
        assert torch.equal(z, y) and torch.equal(h, last)
        assert torch.equal(c.out, want) and torch.equal(g, dh0)


def test_same_inputs_same_bits_and_streams():
    """Calls on a stream of their own; two runs give the same bits (sums in a fixed order)."""
    c = Case(300, 40, 96, torch.bfloat16, 0.02, True, seed=16)
    saved = c.rc.saved()
    a = (*c.forward(saved), *c.backward(saved), c.out.clone())
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        b = (*c.forward(saved), *c.backward(saved), c.out.clone())
    s.synchronize()
    for p, q in zip(a, b):
        assert torch.equal(p, q)


def test_rows_past_four_gigabytes():
    """Rows whose offsets pass 32 bits, in elements and in bytes."""
    T, B, D = 9, 2, 64
    c = Case(T, B, D, torch.bfloat16, seed=17)
    y, last = c.forward()
    st = 300_000_000                    # elements between steps: 4.8 GB end to end
    big = torch.empty((T - 1) * st + B * 3 * D, dtype=torch.bfloat16, device="cuda")
    far = big.as_strided((T, B, 3 * D), (st, 3 * D, 1))
    far.copy_(c.gates)
    out = torch.empty_like(y)
    tp.recur_forward(c.rc, *c.split(far), out, c.work, h0=dev(c.h0))
    torch.cuda.synchronize()
    assert torch.equal(out, y)


def test_graph_replays():
    """Forward and backward captured in a HIP graph and replayed on new inputs."""
    c = Case(130, 4, 64, torch.float32, 0.05, seed=18)
    saved = c.rc.saved()
    y, last = torch.empty(130, 4, 64, device="cuda"), torch.empty(4, 64, device="cuda")
    dlam, dh0 = torch.empty(64, device="cuda"), torch.empty(4, 64, device="cuda")
    h0, dh = dev(c.h0), dev(c.dh)

    def both():
        tp.recur_forward(c.rc, *c.split(c.gates), y, c.work, h0=h0, h_last=last, saved=saved)
        tp.recur_backward(c.rc, *c.split(c.gates), saved, c.dy, *c.split(c.out), dlam, c.work,
                          dh_last=dh, dh0=dh0)

    both()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for k in range(3):
        c.gates.normal_(generator=torch.Generator("cuda").manual_seed(k))
        both()
        want = [t.clone() for t in (y, last, dlam, dh0, c.out)]
        for t in (y, last, dlam, dh0, c.out):
            t.fill_(7.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for p, q in zip((y, last, dlam, dh0, c.out), want):
            assert torch.equal(p, q)


def test_refusals():
    c = Case(4, 2, 64, torch.float32, seed=19)
    x, r, i = c.split(c.gates)
    y = torch.empty(4, 2, 64, device="cuda")
    with pytest.raises(tp.TPError) as e:
        tp.recur_forward(c.rc, x, r, i, y, c.work[:16])
    assert e.value.code == tp.TP_EINVAL and "workspace" in str(e.value)
    with pytest.raises(tp.TPError) as e:
        tp.recur_forward(c.rc, x, r, i, None, c.work)
    assert "no output" in str(e.value)
    with pytest.raises(tp.TPError) as e:    # rows of an output on one another
        tp.recur_forward(c.rc, x, r, i, y[:1].expand(4, 2, 64), c.work)
    assert "overlap" in str(e.value)
    with pytest.raises(AssertionError):
        tp.recur_forward(c.rc, x.bfloat16(), r, i, y, c.work)
