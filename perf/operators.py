"""Performance cases of the operators of a policy with memory: a gated linear recurrence over bars
(whole sequences, their gradients, one bar at a time) and the 4-bit products that feed it.

Sizes are those of this repository's workloads: 64 to 4,096 envs (65,536 in stress), 256 to 390 steps
of a rollout, 63 trading days of minute bars, observations of 31, 301 and 1,001 features (rows padded
to a multiple of 32), hidden widths of 64, 256 and 512.

Kinds of cases
  step    one bar: the recurrence's state moves on by one step
  scan    states of a stored sequence
  train   the same with what the gradients need, and the gradients of everything
  quant   a matrix to 4-bit blocks and back to the values they stand for
  linear  a layer on 4-bit weights: rows of a matrix go to 4 bits, product, bias, activation
  wgrad   a layer's weight gradient: both operands go to 4 bits along the rows, product over the rows
"""

import math

import torch

own = False
DEV = "cuda"
MINUTES = 390                       # bars of a trading day


# --------------------------------------------------------------------------
# the cases
# --------------------------------------------------------------------------

def listed():
    return [
        # One bar of a live loop: 64 accounts, 512 channels.  Latency.
        dict(name="step-bar", kind="step", B=64, D=512, dtype="bf16"),
        # One bar of the stress workload's 65,536 envs.
        dict(name="step-envs", kind="step", B=65536, D=512, dtype="bf16"),
        # A backtest of one account: 63 trading days of minute bars in one sequence.
        dict(name="scan-account", kind="scan", T=63 * MINUTES, B=1, D=512, dtype="bf16",
             ragged=False, ends=0.0),
        # A day of minute bars of 4,096 envs (the headline rollout), some episodes ending inside.
        dict(name="scan-minute", kind="scan", T=MINUTES, B=4096, D=512, dtype="bf16",
             ragged=False, ends=1 / 256),
        # The smallest training step (tiny): 64 envs, 256 steps, 64 channels.
        dict(name="train-tiny", kind="train", T=256, B=64, D=64, dtype="f32", ragged=False,
             ends=1 / 64),
        # A year of daily bars of 1,024 envs in fp32, sequences of unequal length (some empty).
        dict(name="train-daily", kind="train", T=252, B=1024, D=256, dtype="f32", ragged=True,
             ends=0.0),
        # The headline rollout's training step.
        dict(name="train-minute", kind="train", T=MINUTES, B=4096, D=512, dtype="bf16",
             ragged=False, ends=1 / 256),
        # Observations of 65,536 envs to 4 bits.
        dict(name="quant-envs", kind="quant", rows=65536, K=1001, dtype="bf16", turned=False),
        # Gradients of the gates, turned: blocks of 32 run along the rows in memory.
        dict(name="quant-turned", kind="quant", rows=1536, K=11 * 1001, dtype="f32", turned=True),
        # The three gates of 64 accounts from one bar's observation.
        dict(name="linear-bar", kind="linear", M=64, N=1536, K=1001, dtype="bf16", act="none"),
        # The same for 65,536 envs.
        dict(name="linear-envs", kind="linear", M=65536, N=1536, K=1001, dtype="bf16", act="none"),
        # The gates' weight gradient over 16 steps of 4,096 envs.
        dict(name="wgrad-minute", kind="wgrad", rows=65536, N=1536, K=1001, dtype="bf16"),
    ]


def _log(rng, lo, hi):
    """An integer spread evenly over the logarithm of [lo, hi]."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _width(rng):
    """Channels: the networks' widths, and others from 64 to 768."""
    return rng.choice([64, 128, 256, 512, 512, 768, _log(rng, 64, 768)])


def _features(rng):
    """Features of an observation: 1 + 2 n + n I of a market, or a hidden width."""
    n = _log(rng, 5, 100)
    return rng.choice([31, 301, 1001, 256, 512, 1024, 1 + 2 * n + n * rng.choice([4, 5, 8])])


def draw(rng):
    kind = rng.choice(["step", "scan", "scan", "train", "train", "quant", "linear", "linear",
                       "wgrad"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if kind == "step":
        return dict(kind=kind, B=_log(rng, 1, 65536), D=_width(rng), dtype=dtype)
    if kind in ("scan", "train"):
        D = _width(rng)
        T = _log(rng, 1, 63 * MINUTES if kind == "scan" else 2520)
        most = MINUTES * 4096 * 512 // (2 if dtype == "f32" else 1)
        B = _log(rng, 1, max(1, min(4096, most // (T * D))))
        return dict(kind=kind, T=T, B=B, D=D, dtype=dtype, ragged=rng.random() < 0.3,
                    ends=rng.choice([0.0, 1 / 64, 1 / 256]))
    if kind == "quant":
        return dict(kind=kind, rows=_log(rng, 1, 32768), K=_features(rng), dtype=dtype,
                    turned=rng.random() < 0.3)
    N = rng.choice([100, 256, 512, 768, 1536, _log(rng, 5, 1536)])
    if kind == "linear":
        return dict(kind=kind, M=_log(rng, 1, 65536), N=N, K=_features(rng), dtype=dtype,
                    act=rng.choice(["none", "tanh"]))
    return dict(kind=kind, rows=_log(rng, 64, 65536), N=N, K=_features(rng), dtype=dtype)


# --------------------------------------------------------------------------
# sizes
# --------------------------------------------------------------------------

def _size(c):
    return 2 if c["dtype"] == "bf16" else 4


def _torch(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def work(c):
    kind, z = c["kind"], _size(c)
    if kind == "step":                      # x, r, i in, y out, the state in and out
        n = c["B"] * c["D"]
        return dict(bytes=n * (4 * z + 8) + 4 * c["D"], flops=25 * n)
    if kind in ("scan", "train"):
        n, edge = c["T"] * c["B"] * c["D"], 4 * c["B"] * c["D"]
        flags = (c["T"] * c["B"] if c["ends"] else 0) + (4 * c["B"] if c["ragged"] else 0)
        if kind == "scan":                  # x, r, i in, y out, the first and last states
            return dict(bytes=4 * n * z + 2 * edge + 4 * c["D"] + flags, flops=25 * n)
        # x, r, i, dy in, y, dx, dr, di out
        return dict(bytes=8 * n * z + 4 * edge + 8 * c["D"] + flags, flops=70 * n)
    if kind == "quant":                     # in, 4 bits and a scale of 8 for each 32, out again
        n = c["rows"] * c["K"]
        return dict(bytes=n * (2 * z + 0.5) + c["rows"] * -(-c["K"] // 32), flops=6 * n)
    four = lambda rows, k: rows * (k / 2 + -(-k // 32))  # noqa: E731
    if kind == "linear":
        return dict(bytes=c["M"] * c["K"] * z + four(c["N"], c["K"]) + 4 * c["N"] +
                    c["M"] * c["N"] * z, flops=2 * c["M"] * c["N"] * c["K"])
    return dict(bytes=c["rows"] * (c["N"] + c["K"]) * z + 4 * c["N"] * c["K"],
                flops=2 * c["rows"] * c["N"] * c["K"])


# --------------------------------------------------------------------------
# inputs
# --------------------------------------------------------------------------

def _gen(seed, stream):
    g = torch.Generator(device=DEV)
    g.manual_seed((seed * 1_000_003 + stream) % (1 << 62))
    return g


def _normal(seed, stream, shape, dtype=torch.float32, scale=1.0):
    t = torch.empty(shape, dtype=dtype, device=DEV).normal_(generator=_gen(seed, stream))
    return t.mul_(scale) if scale != 1.0 else t


def _decays(seed, D):
    """lambda of channels whose state fades by a factor of 0.9 to 0.9995 a step at an open gate of
    one half: memories of 10 to 2,000 bars."""
    a = 1.0 - 10.0 ** -(1.0 + 2.3 * torch.rand(D, generator=_gen(seed, 1), device=DEV))
    return torch.log(torch.expm1(-torch.log(a) / 4.0))


def _observations(c, rows, seed):
    """Observation rows [rows][ld], ld = K padded to a multiple of 32 as the env writes them: N(0,1)
    indicators after balance, prices and holdings of the market's scales."""
    K = c["K"]
    obs = _normal(seed, 2, (rows, -(-K // 32) * 32), _torch(c))
    n = K // 10                             # 1 + 2 n + 8 n features
    if n:
        g = _gen(seed, 3)
        obs[:, 0] = torch.rand(rows, generator=g, device=DEV) + 0.5
        obs[:, 1:1 + n] = (torch.rand(rows, n, generator=g, device=DEV) * 180 + 20) / 128
        obs[:, 1 + n:1 + 2 * n] = torch.randint(0, 300, (rows, n), generator=g, device=DEV) / 128
    return obs[:, :K]


def _sequence(c, seed):
    """Gates as one product writes them, [T][B][3 D]: x, r, i are views of it."""
    T, B, D = c["T"], c["B"], c["D"]
    s = dict(kind=c["kind"], c=c, lam=_decays(seed, D), done=None, lens=None,
             gates=_normal(seed, 4, (T, B, 3 * D), _torch(c)), h0=_normal(seed, 5, (B, D)))
    if c["ends"]:
        s["done"] = (torch.rand(T, B, generator=_gen(seed, 6), device=DEV) < c["ends"]).byte()
    if c["ragged"]:
        s["lens"] = torch.randint(0, T + 1, (B,), generator=_gen(seed, 7), device=DEV,
                                  dtype=torch.int32)
    if c["kind"] == "train":
        s["dy"] = _normal(seed, 8, (T, B, D), _torch(c))
        s["dh_last"] = _normal(seed, 9, (B, D))
    return s


def _inputs(c, seed):
    kind = c["kind"]
    if kind == "step":
        B, D = c["B"], c["D"]
        return dict(kind=kind, c=c, lam=_decays(seed, D), h=_normal(seed, 5, (B, D)),
                    gates=_normal(seed, 4, (B, 3 * D), _torch(c)),
                    done=(torch.rand(B, generator=_gen(seed, 6), device=DEV) < 1 / 256).byte())
    if kind in ("scan", "train"):
        return _sequence(c, seed)
    if kind == "quant":
        if c["turned"]:
            x = _normal(seed, 2, (c["K"], c["rows"]), _torch(c)).t()
        else:
            x = _observations(c, c["rows"], seed)
        return dict(kind=kind, c=c, x=x)
    if kind == "linear":
        K = c["K"]
        return dict(kind=kind, c=c, x=_observations(c, c["M"], seed),
                    w=_normal(seed, 10, (c["N"], K), scale=K ** -0.5),
                    bias=_normal(seed, 11, (c["N"],), scale=0.1))
    return dict(kind=kind, c=c, x=_observations(c, c["rows"], seed),
                dg=_normal(seed, 12, (c["rows"], c["N"]), _torch(c), 1e-3))


def prepare(c, seed):
    s = _inputs(c, seed)
    if own:
        _buffers(s)                         # descriptors, 4-bit weights, outputs, workspaces
    elif c["kind"] == "linear":
        s["w"] = _four_bits(s["w"])         # the layer keeps its weights in 4 bits
    return s


def _views(t, D):
    return t[..., :D], t[..., D:2 * D], t[..., 2 * D:]


# --------------------------------------------------------------------------
# the plain forms
# --------------------------------------------------------------------------

def _sigmoid(x):
    return 1.0 / (1.0 + torch.exp(-x))


def _softplus(x):
    return torch.clamp(x, min=0.0) + torch.log1p(torch.exp(-torch.abs(x)))


def _coefficients(x, r, i, lam):
    """L = log a, a, beta and the gated input iota x, in fp32."""
    L = _sigmoid(r.float()) * (-8.0 * _softplus(lam))
    return L, torch.exp(L), torch.sqrt(-torch.expm1(2.0 * L)), _sigmoid(i.float()) * x.float()


def _scan(a, u):
    """h_t = a_t h_{t-1} + u_t with h_{-1} = 0, in place of u: step by step where a step fills the
    GPU, else log2(T) rounds over all steps."""
    T = a.shape[0]
    if a[0].numel() >= 1 << 15:
        for t in range(1, T):
            u[t].addcmul_(a[t], u[t - 1])
        return u
    a, k = a.clone(), 1
    while k < T:
        u[k:] = u[k:] + a[k:] * u[:-k]
        a[k:] = a[k:] * a[:-k]
        k *= 2
    return u


def _masks(s):
    """valid [T][B][1] (or None) and open [T][B][1]: the state goes on after step t."""
    T, B = s["c"]["T"], s["c"]["B"]
    valid = None
    if s["lens"] is not None:
        valid = (torch.arange(T, device=DEV)[:, None] < s["lens"][None])[:, :, None]
    opened = torch.ones(T, B, 1, device=DEV)
    if s["done"] is not None:
        opened = (s["done"] == 0).float()[:, :, None]
    return valid, opened


def _forward(s):
    c = s["c"]
    x, r, i = _views(s["gates"], c["D"])
    L, a, beta, q = _coefficients(x, r, i, s["lam"])
    valid, opened = _masks(s)
    u = beta * q
    if valid is not None:                   # past its end a sequence's state stays as it is
        u = torch.where(valid, u, 0.0)
        a = torch.where(valid, a, 1.0)
        opened = torch.where(valid, opened, 1.0)
    carry = a.clone()                       # from the state after step t - 1 to the one after t
    carry[1:] *= opened[:-1]
    u[0] += carry[0] * s["h0"]
    h = _scan(carry, u)
    h_last = h[-1] * opened[-1]
    y = h if valid is None else torch.where(valid, h, 0.0)
    return (L, a, beta, q, carry, opened, valid, h), y.to(_torch(c)), h_last


def _gradients(s, kept):
    c = s["c"]
    x, r, i = _views(s["gates"], c["D"])
    L, a, beta, q, carry, opened, valid, h = kept
    dy = s["dy"].float()
    if valid is not None:
        dy = torch.where(valid, dy, 0.0)
    g = dy.clone()
    g[-1] += opened[-1] * s["dh_last"]
    # the same recurrence from the last step to the first
    back = torch.cat([torch.ones_like(carry[:1]), carry.flip(0)[:-1]])
    g = _scan(back, g.flip(0)).flip(0)
    del back, dy
    dh0 = carry[0] * g[0]
    hprev = torch.cat([s["h0"][None], h[:-1] * opened[:-1]])
    iota, rho = _sigmoid(i.float()), _sigmoid(r.float())
    w = g * (L * a * hprev - q * a * a * (L / beta))
    dx, di, dr = g * beta * iota, g * beta * q * (1.0 - iota), w * (1.0 - rho)
    if valid is not None:
        dx, di, dr, w = (torch.where(valid, v, 0.0) for v in (dx, di, dr, w))
    dlam = w.sum(dim=(0, 1)) * (_sigmoid(s["lam"]) / _softplus(s["lam"]))
    return torch.cat([dx, dr, di], dim=2).to(_torch(c)), dlam, dh0


def _power(e):
    """2^e of whole e in [-126, 127], from its bits."""
    return ((e + 127) << 23).view(torch.float32)


def _four_bits(x):
    """The values of x [rows][K] in blocks of 32 along K: E2M1 elements (0, 1/2, 1, 3/2, 2, 3, 4,
    6), nearest, ties to the even code, times 2^(floor(log2 of the block's largest) - 2)."""
    R, K = x.shape
    v = torch.zeros(R, -(-K // 32), 32, device=DEV)
    v.view(R, -1)[:, :K] = x.float()
    _, e = torch.frexp(v.abs().amax(dim=2, keepdim=True))
    e = torch.clamp(e - 3, -126, 126)
    v = v * _power(-e)
    m = v.abs()
    code = ((m > 0.25).byte() + (m >= 0.75) + (m > 1.25) + (m >= 1.75) + (m > 2.5) + (m >= 3.5) +
            (m > 5.0))
    grid = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=DEV)
    q = torch.copysign(grid[code.int()], v) * _power(e)
    return q.view(R, -1)[:, :K]


def _plain(s):
    kind, c = s["kind"], s["c"]
    if kind == "step":
        x, r, i = _views(s["gates"], c["D"])
        _, a, beta, q = _coefficients(x, r, i, s["lam"])
        h = a * s["h"] + beta * q
        return dict(y=h.to(_torch(c)), h=torch.where(s["done"][:, None] != 0, 0.0, h))
    if kind == "scan":
        _, y, h_last = _forward(s)
        return dict(y=y, h_last=h_last)
    if kind == "train":
        kept, y, h_last = _forward(s)
        dgates, dlam, dh0 = _gradients(s, kept)
        return dict(y=y, h_last=h_last, dgates=dgates, dlam=dlam, dh0=dh0)
    if kind == "quant":
        return _four_bits(s["x"]).to(_torch(c))
    if kind == "linear":
        z = _four_bits(s["x"]) @ s["w"].t() + s["bias"]
        return (torch.tanh(z) if c["act"] == "tanh" else z).to(_torch(c))
    return _four_bits(s["dg"].t()) @ _four_bits(s["x"].t()).t()


# --------------------------------------------------------------------------
# the framework's operators
# --------------------------------------------------------------------------

def _buffers(s):
    """What a program keeps between calls: descriptors, 4-bit weights, outputs and workspaces."""
    from paper_2111_05188_amd import tp
    kind, c = s["kind"], s["c"]
    new = lambda *shape, dtype=_torch(c): torch.empty(shape, dtype=dtype, device=DEV)  # noqa: E731
    if kind == "step":
        s["y"], s["h_next"] = new(c["B"], c["D"]), new(c["B"], c["D"], dtype=torch.float32)
    elif kind in ("scan", "train"):
        T, B, D = c["T"], c["B"], c["D"]
        s["rc"] = rc = tp.RecurT(s["lam"], T, B, _torch(c), done=s["done"], lens=s["lens"])
        s["work"], s["y"] = rc.workspace(), new(T, B, D)
        s["h_last"] = new(B, D, dtype=torch.float32)
        if kind == "train":
            s["saved"], s["dgates"] = rc.saved(), new(T, B, 3 * D)
            s["dlam"], s["dh0"] = new(D, dtype=torch.float32), new(B, D, dtype=torch.float32)
    elif kind == "quant":
        s["four"] = tp.Mx4T.empty(c["rows"], c["K"])
        s["y"] = new(c["rows"], c["K"])
    elif kind == "linear":
        s["four"] = tp.mx4_quantize(s["w"])
        s["y"], s["work"] = new(c["M"], c["N"]), tp.mx4_workspace(c["M"], c["N"], c["K"])
    else:
        s["a"] = tp.Mx4T.empty(c["N"], c["rows"])
        s["b"] = tp.Mx4T.empty(c["K"], c["rows"])
        s["y"] = new(c["N"], c["K"], dtype=torch.float32)
        s["work"] = tp.mx4_workspace(c["N"], c["K"], c["rows"])


def _run(s):
    from paper_2111_05188_amd import tp
    kind, c = s["kind"], s["c"]
    if kind == "step":
        tp.recur_step(*_views(s["gates"], c["D"]), s["lam"], s["h"], s["h_next"], s["y"],
                      done=s["done"])
        return dict(y=s["y"], h=s["h_next"])
    if kind == "scan":
        tp.recur_forward(s["rc"], *_views(s["gates"], c["D"]), s["y"], s["work"], h0=s["h0"],
                         h_last=s["h_last"])
        return dict(y=s["y"], h_last=s["h_last"])
    if kind == "train":
        gates = _views(s["gates"], c["D"])
        tp.recur_forward(s["rc"], *gates, s["y"], s["work"], h0=s["h0"], h_last=s["h_last"],
                         saved=s["saved"])
        tp.recur_backward(s["rc"], *gates, s["saved"], s["dy"], *_views(s["dgates"], c["D"]),
                          s["dlam"], s["work"], dh_last=s["dh_last"], dh0=s["dh0"])
        return {k: s[k] for k in ("y", "h_last", "dgates", "dlam", "dh0")}
    if kind == "quant":
        tp.mx4_quantize(s["x"], s["four"])
        tp.mx4_dequantize(s["four"], s["y"])
        return s["y"]
    if kind == "linear":
        act = tp.TP_ACT_TANH if c["act"] == "tanh" else tp.TP_ACT_NONE
        tp.mx4_linear(s["x"], s["four"], s["y"], bias=s["bias"], act=act, work=s["work"])
        return s["y"]
    tp.mx4_quantize(s["dg"].t(), s["a"])
    tp.mx4_quantize(s["x"].t(), s["b"])
    tp.mx4_matmul(s["a"], s["b"], s["y"], work=s["work"])
    return s["y"]


def run(s):
    return _run(s) if own else _plain(s)


# --------------------------------------------------------------------------
# the definitions in 64 bits
# --------------------------------------------------------------------------

def _exact_states(gates, lam, h, done, lens):
    """States after each step by the definition, one step at a time; y and the last state."""
    x, r, i = _views(gates, lam.shape[0])
    L = -8.0 * torch.nn.functional.softplus(lam) * torch.sigmoid(r)
    a, u = torch.exp(L), torch.sqrt(-torch.expm1(2.0 * L)) * torch.sigmoid(i) * x
    ys = []
    for t in range(x.shape[0]):
        new = a[t] * h + u[t]
        after = new if done is None else new * (done[t][:, None] == 0)
        if lens is not None:
            live = (t < lens)[:, None]
            new, after = new * live, torch.where(live, after, h)
        ys.append(new)
        h = after
    return torch.stack(ys), h


def _exact_sequence(s):
    """A part of the envs at a time; gradients by differentiating the definition."""
    c, train = s["c"], s["c"]["kind"] == "train"
    T, B, D = c["T"], c["B"], c["D"]
    part = max(1, (80_000_000 if train else 200_000_000) // (T * D))
    outs = []
    dlam = torch.zeros(D, dtype=torch.float64, device=DEV)
    for b in range(0, B, part):
        e = slice(b, b + part)
        gates, lam, h0 = s["gates"][:, e].double(), s["lam"].double(), s["h0"][e].double()
        done = None if s["done"] is None else s["done"][:, e]
        lens = None if s["lens"] is None else s["lens"][e]
        with torch.set_grad_enabled(train):
            for v in (gates, lam, h0):
                v.requires_grad_(train)
            y, h = _exact_states(gates, lam, h0, done, lens)
            if train:
                loss = (y * s["dy"][:, e].double()).sum() + (h * s["dh_last"][e].double()).sum()
                loss.backward()
        outs.append((y.detach(), h.detach()) + ((gates.grad, h0.grad) if train else ()))
        dlam += lam.grad if train else 0.0
        del gates, h0, y, h
    y, h, *more = zip(*outs)
    out = dict(y=torch.cat(y, 1), h_last=torch.cat(h))
    if train:
        out.update(dgates=torch.cat(more[0], 1), dlam=dlam, dh0=torch.cat(more[1]))
    return out


def _exact_four_bits(x):
    """Rounding to a multiple of 1/2, 1 or 2 by magnitude, of x / scale in 64 bits."""
    R, K = x.shape
    v = torch.zeros(R, -(-K // 32) * 32, dtype=torch.float64, device=DEV)
    v[:, :K] = x.double()
    v = v.view(R, -1, 32)
    _, e = torch.frexp(v.abs().amax(dim=2, keepdim=True))
    scale = ((torch.clamp(e.long() - 3, -127, 127) + 1023) << 52).view(torch.float64)
    m = v / scale
    grain = torch.where(m.abs() < 2.0, 0.5, torch.where(m.abs() < 4.0, 1.0, 2.0)).double()
    q = torch.clamp(torch.round(m / grain) * grain, -6.0, 6.0) * scale
    return q.view(R, -1)[:, :K]


def exact(c, seed):
    kind, s = c["kind"], _inputs(c, seed)
    if kind == "step":
        y, h = _exact_states(s["gates"][None].double(), s["lam"].double(), s["h"].double(),
                             s["done"][None], None)
        return dict(y=y[0], h=h)
    if kind in ("scan", "train"):
        return _exact_sequence(s)
    if kind == "quant":
        return _exact_four_bits(s["x"])
    if kind == "linear":
        z = _exact_four_bits(s["x"]) @ _exact_four_bits(s["w"]).t() + s["bias"].double()
        return torch.tanh(z) if c["act"] == "tanh" else z
    return _exact_four_bits(s["dg"].t()) @ _exact_four_bits(s["x"].t()).t()
