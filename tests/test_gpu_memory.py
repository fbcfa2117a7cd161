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


def clobber(stream, *sizes):
    """The current stream's next memory of these sizes in bytes, filled with other bytes while
    `stream` has its work before it."""
    junk = [torch.full((n,), 0xEE, dtype=torch.uint8, device="cuda") for n in sizes for _ in range(2)]
    torch.cuda.current_stream().synchronize()
    assert not stream.query()
    return junk


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_calls_on_a_stream_of_their_own(dtype):
    """Calls on a stream that is busy, while the current stream goes on with its own work: the
    layer's temporaries, copies and buffers of another size are in the order of the calls."""
    S, D, T, B = 301, 64, 40, 30
    g = torch.Generator("cuda").manual_seed(8)
    obs = torch.randn(B, T, 320, generator=g, device="cuda").transpose(0, 1)    # not in one piece
    dy = torch.randn(T, B, D, generator=g, device="cuda").to(dtype)
    layer = memory.MemoryLayer.init(S, D, 7, dtype)
    size = torch.empty(0, dtype=dtype).element_size()

    def calls(stream):
        h = torch.zeros(B, D, device="cuda")
        layer.encode(obs)                       # buffers from before, of the current stream
        torch.cuda.synchronize()
        own = stream is not None
        if own:
            with torch.cuda.stream(stream):
                torch.cuda._sleep(500_000_000)     # a fifth of a second
        out, kept = [], []
        for t in range(3):
            out.append(layer.step(obs[t], h, stream=stream))
            if own:
                kept += clobber(stream, 3 * B * D * size, B * D * size)
        if own:
            torch.cuda._sleep(1_000_000)        # the current stream is busy too
        out += [*layer.encode(obs, stream=stream), *layer.gradients(dy, stream=stream)]
        kept_sizes = [t.numel() * t.element_size() for t in
                      (layer.gates, layer.dgates, layer.saved, layer.work, layer.workW,
                       layer.dg4.data, layer.obs4.data, layer.work1)]
        out += layer.encode(obs[:20], stream=stream)
        out.append(layer.step(obs[0, :20], h[:20], stream=stream))
        if own:
            kept += clobber(stream, *kept_sizes)
            stream.synchronize()
        torch.cuda.synchronize()
        return [t.clone() for t in (*out, h)]

    want = calls(None)
    for t, p in zip(want, calls(torch.cuda.Stream())):
        assert torch.equal(t, p)


def test_streams_take_turns():
    """Calls of one layer on two streams without a wait between them run in their order."""
    layer = memory.MemoryLayer.init(31, 64, 9, torch.float32)
    obs = torch.randn(2, 50, 8, 32, generator=torch.Generator("cuda").manual_seed(10), device="cuda")
    dy = torch.ones(50, 8, 64, device="cuda")
    want = []
    for o in obs:
        layer.encode(o)
        want.append([t.clone() for t in layer.gradients(dy)])
    torch.cuda.synchronize()
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    with torch.cuda.stream(a):
        torch.cuda._sleep(500_000_000)     # a fifth of a second
    layer.encode(obs[0], stream=a)
    got = layer.gradients(dy, stream=b)
    with torch.cuda.stream(b):
        first = [t.clone() for t in got]
    layer.encode(obs[1], stream=a)
    second = layer.gradients(dy, stream=a)
    torch.cuda.synchronize()
    for p, q in zip(want, (first, second)):
        for t, u in zip(p, q):
            assert torch.equal(t, u)


def test_step_in_a_graph():
    """One bar captured and replayed on new observations, after steps outside the capture."""
    layer = memory.MemoryLayer.init(31, 64, 11)
    g = torch.Generator("cuda").manual_seed(12)
    obs, h = torch.randn(8, 32, generator=g, device="cuda"), torch.zeros(8, 64, device="cuda")
    layer.step(obs, h)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = layer.step(obs, h)
    for _ in range(3):
        obs.normal_(generator=g)
        h.fill_(0.5)
        want = layer.step(obs, h).clone()
        state = h.clone()
        h.fill_(0.5)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want) and torch.equal(h, state)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("junk", [1e6, float("nan"), float("inf")])
def test_nothing_past_a_sequences_end_matters(dtype, junk):
    """Ragged lengths: whatever the observations hold past them, every result is that of zeros
    there, and W's gradient the product over the rows that the sequences have."""
    T, B, S, D = 37, 9, 70, 48
    g = torch.Generator("cuda").manual_seed(13)
    lens = torch.tensor([0, T, 1, 5, 36, 20, 31, 12, 17], dtype=torch.int32, device="cuda")
    past = torch.arange(T, device="cuda")[:, None] >= lens
    clean = torch.randn(T, B, 96, generator=g, device="cuda").to(dtype).masked_fill(past[..., None], 0.0)
    dirty = clean.masked_fill(past[..., None], junk)
    done = (torch.rand(T, B, generator=g, device="cuda") < 0.1).byte()
    h0, dh = torch.randn(2, B, D, generator=g, device="cuda")
    dy = torch.randn(T, B, D, generator=g, device="cuda").to(dtype)
    layer, res = memory.MemoryLayer.init(S, D, 14, dtype), []
    for obs in (clean, dirty):
        out = [*layer.encode(obs, done, lens, h0), *layer.gradients(dy, dh)]
        torch.cuda.synchronize()
        res.append([t.clone() for t in (*out, layer.dgates)])
    for p, q in zip(*res):
        assert torch.isfinite(p).all() and torch.equal(p, q)
    a = mx4.values(host(layer.dgates.reshape(T * B, -1)).T)
    b = mx4.values(host(clean.reshape(T * B, -1)[:, :S]).T)
    want, mass = mx4.product(a, b)
    assert (np.abs(host(layer.dW) - want) <= (T * B / 64 + 8) * 2.0 ** -23 * mass).all()
    assert (layer.dgates[past] == 0).all()


@pytest.mark.parametrize("dtype,tol", [(torch.float32, 3e-5), (torch.bfloat16, 3e-5 + 2.0 ** -8)])
def test_states_and_gradients_of_a_layer(dtype, tol):
    """Both types, with first states, last states' gradients, episode ends and lengths: each part
    against 64 bits on what the part before it stored."""
    T, B, S, D = 60, 5, 301, 40
    rng = np.random.default_rng(15)
    dev = lambda v, dt: torch.from_numpy(np.asarray(v)).cuda().to(dt)  # noqa: E731
    obs = dev(rng.normal(size=(T, B, 320)), dtype)
    done, lens = (rng.random((T, B)) < 0.05).astype(np.uint8), np.array([60, 0, 7, 33, 59], np.int32)
    h0, dh, dy = rng.normal(size=(B, D)), rng.normal(size=(B, D)), rng.normal(size=(T, B, D))
    layer = memory.MemoryLayer.init(S, D, 16, dtype)
    y, last = layer.encode(obs, dev(done, torch.uint8), dev(lens, torch.int32), dev(h0, torch.float32))
    dy = dev(dy, dtype)
    dW, dlam, dh0 = layer.gradients(dy, dev(dh, torch.float32))
    torch.cuda.synchronize()
    x, w = mx4.values(host(obs.reshape(T * B, -1)[:, :S])), mx4.values(host(layer.W))
    want, mass = mx4.product(x, w)
    off = np.abs(host(layer.gates).reshape(T * B, -1) - want)
    assert (off <= (S / 64 + 8) * 2.0 ** -23 * mass +
            (2.0 ** -8 * np.abs(want) if dtype == torch.bfloat16 else 0.0)).all()
    parts, lam = [host(v) for v in layer.parts(layer.gates)], host(layer.lam)
    h0, dh = h0.astype(np.float32).astype(np.float64), dh.astype(np.float32).astype(np.float64)
    wy, wl = recur.forward(*parts, lam, h0, done, lens)
    rms_close(y, wy, tol)
    rms_close(last, wl, 3e-5)
    dx, dr, di, wlam, wh0, mass = recur.backward(*parts, lam, host(dy), dh, h0, done, lens)
    rms_close(layer.dgates, np.concatenate([dx, dr, di], axis=2), tol)
    assert (np.abs(host(dlam) - wlam) <= 3e-5 * mass + 1e-16).all()
    rms_close(dh0, wh0, 3e-5)
    seen = (np.arange(T)[:, None] < lens).reshape(-1, 1)
    want, mass = mx4.product(mx4.values(host(layer.dgates).reshape(T * B, -1).T),
                             mx4.values(np.where(seen, host(obs).reshape(T * B, -1)[:, :S], 0.0).T))
    assert (np.abs(host(dW) - want) <= (T * B / 64 + 8) * 2.0 ** -23 * mass).all()
