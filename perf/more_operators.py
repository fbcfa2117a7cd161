"""Performance cases of the operators of a policy made of blocks with a matrix memory: the gated
delta rule over bars (whole sequences, their gradients, one bar at a time), the norms around a
block with its gate and residual scale, and the clipped policy loss with a KL term.

Sizes are those of this repository's workloads: 64 to 4,096 envs, 252 to 390 steps of a rollout, 63
trading days of minute bars, 30 and 100 stocks, widths of 64 to 512 channels in heads of 32 to 128.

Kinds of cases
  step    one bar: the matrix states of all heads move on by one step
  scan    outputs and last states of stored sequences
  train   the same with what the gradients need, and the gradients of everything
  norm    a block's output normed, gated, scaled and added to the residual stream, and the norm
          that the next block reads
  normgrad  the same and its gradients
  loss    the clipped policy loss of a Gaussian policy with KL to the policy that acted, and its
          gradient
"""

import math

import torch

own = False
DEV = "cuda"
MINUTES = 390                       # bars of a trading day
EPS = 1e-6                          # of the norms, and of the keys' and queries' lengths


# --------------------------------------------------------------------------
# the cases
# --------------------------------------------------------------------------

def listed():
    return [
        # One bar of a live loop: 64 accounts, 8 heads.  Latency.
        dict(name="step-bar", kind="step", B=64, H=8, dk=64, dv=64, dtype="bf16"),
        # One bar of a rollout's 4,096 envs.
        dict(name="step-envs", kind="step", B=4096, H=8, dk=64, dv=64, dtype="bf16"),
        # A backtest of one account: 63 trading days of minute bars in one sequence, wide heads.
        dict(name="scan-account", kind="scan", T=63 * MINUTES, B=1, H=4, dk=128, dv=128,
             dtype="bf16", ragged=False, ends=0.0),
        # A day of minute bars of 4,096 envs (the headline rollout), some episodes ending inside.
        dict(name="scan-minute", kind="scan", T=MINUTES, B=4096, H=4, dk=64, dv=64, dtype="bf16",
             ragged=False, ends=1 / 256),
        # The smallest training step (tiny): 64 envs, 64 steps, two narrow heads.
        dict(name="train-tiny", kind="train", T=64, B=64, H=2, dk=32, dv=32, dtype="f32",
             ragged=False, ends=1 / 64),
        # A year of daily bars of 1,024 envs in fp32, sequences of unequal length (some empty).
        dict(name="train-daily", kind="train", T=252, B=1024, H=4, dk=64, dv=64, dtype="f32",
             ragged=True, ends=0.0),
        # The training step of a day of minute bars, half the headline rollout's envs at a time.
        dict(name="train-minute", kind="train", T=MINUTES, B=2048, H=4, dk=64, dv=64,
             dtype="bf16", ragged=False, ends=1 / 256),
        # One bar of a live loop through a block's norms.  Latency.
        dict(name="norm-bar", kind="norm", rows=64, D=512, groups=8, dtype="bf16"),
        # The same over a day of minute bars of 4,096 envs.
        dict(name="norm-minute", kind="norm", rows=MINUTES * 4096, D=256, groups=4, dtype="bf16"),
        # Norms of a year of daily bars of 1,024 envs with their gradients, one norm over an odd
        # row.
        dict(name="normgrad-daily", kind="normgrad", rows=252 * 1024, D=301, groups=1,
             dtype="f32"),
        # The policy loss of a year of daily bars of 1,024 envs, 30 stocks, unequal lengths.
        dict(name="loss-daily", kind="loss", T=252, B=1024, n=30, dtype="f32", ragged=True),
        # The policy loss of the headline rollout, 100 stocks.
        dict(name="loss-minute", kind="loss", T=MINUTES, B=4096, n=100, dtype="bf16",
             ragged=False),
    ]


def _log(rng, lo, hi):
    """An integer spread evenly over the logarithm of [lo, hi]."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _heads(rng):
    """Heads, and channels of a head's keys and values."""
    d = rng.choice([32, 64, 64, 64, 128, _log(rng, 16, 128)])
    return dict(H=rng.choice([1, 2, 4, 4, 8]), dk=d, dv=rng.choice([d, d, d, _log(rng, 16, 128)]))


def draw(rng):
    kind = rng.choice(["step", "scan", "scan", "train", "train", "train", "norm", "normgrad",
                       "loss"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    half = 2 if dtype == "f32" else 1
    if kind == "step":
        c = dict(kind=kind, B=0, **_heads(rng), dtype=dtype)
        c["B"] = _log(rng, 1, min(4096, 4096 * 8 * 64 * 64 // (c["H"] * 128 * 128)))
        return c
    if kind in ("scan", "train"):
        c = dict(kind=kind, T=0, B=0, **_heads(rng), dtype=dtype, ragged=rng.random() < 0.3,
                 ends=rng.choice([0.0, 1 / 64, 1 / 256]))
        c["T"] = _log(rng, 1, 63 * MINUTES if kind == "scan" else 2520)
        width = c["H"] * max(c["dk"], c["dv"], 64)
        most = MINUTES * (4096 if kind == "scan" else 2048) * 4 * 64 // half
        c["B"] = _log(rng, 1, max(1, min(4096, most // (c["T"] * width))))
        return c
    if kind in ("norm", "normgrad"):
        D = rng.choice([64, 128, 256, 256, 512, 768, 301, _log(rng, 32, 1024)])
        most = MINUTES * 4096 * 256 // half // (2 if kind == "normgrad" else 1)
        return dict(kind=kind, rows=_log(rng, 1, most // D), D=D,
                    groups=rng.choice([1, 4, 8]) if D % 8 == 0 else 1, dtype=dtype)
    n = rng.choice([5, 30, 100, 100, _log(rng, 1, 128)])
    T = _log(rng, 1, MINUTES)
    return dict(kind=kind, T=T, B=_log(rng, 1, max(1, MINUTES * 4096 // half // T)), n=n,
                dtype=dtype, ragged=rng.random() < 0.4)


# --------------------------------------------------------------------------
# sizes
# --------------------------------------------------------------------------

def _size(c):
    return 2 if c["dtype"] == "bf16" else 4


def _torch(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def work(c):
    kind, z = c["kind"], _size(c)
    if kind in ("step", "scan", "train"):
        n, H, dk, dv = c.get("T", 1) * c["B"] * c["H"], c["H"], c["dk"], c["dv"]
        state = 4 * c["B"] * H * dk * dv
        flags = c["B"] if kind == "step" else \
            (c["T"] * c["B"] if c["ends"] else 0) + (4 * c["B"] if c["ragged"] else 0)
        # q, k, v, r, b in, y out, the first and last states; a step decays the state, reads it
        # twice and adds to it
        fwd = n * (2 * dk + 2 * dv + 2) * z + 2 * state + 4 * H + flags
        if kind != "train":
            return dict(bytes=fwd, flops=7 * n * dk * dv)
        # dy in, dq, dk, dv, dr, db out, and the states' gradients
        return dict(bytes=fwd + n * (2 * dk + 2 * dv + 2) * z + 2 * state + 4 * H,
                    flops=21 * n * dk * dv)
    if kind in ("norm", "normgrad"):
        n = c["rows"] * c["D"]
        if kind == "norm":                  # x, y, z in, x', n out
            return dict(bytes=5 * n * z + 12 * c["D"], flops=15 * n)
        # dx', dn in, dx, dy, dz out
        return dict(bytes=10 * n * z + 24 * c["D"], flops=50 * n)
    rows = c["T"] * c["B"]                  # mu, action, the mean that acted, two numbers in; dmu out
    return dict(bytes=rows * (c["n"] * (2 * z + 8) + 8) + (4 * c["B"] if c["ragged"] else 0) +
                12 * c["n"], flops=20 * rows * c["n"])


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


def _decays(seed, H):
    """lambda of heads whose state fades by a factor of 0.9 to 0.9995 a step at an open gate of one
    half: memories of 10 to 2,000 bars."""
    a = 1.0 - 10.0 ** -(1.0 + 2.3 * torch.rand(H, generator=_gen(seed, 1), device=DEV))
    return torch.log(torch.expm1(-torch.log(a) / 4.0))


def _lens(c, seed):
    return torch.randint(0, c["T"] + 1, (c["B"],), generator=_gen(seed, 7), device=DEV,
                         dtype=torch.int32) if c["ragged"] else None


def _delta_inputs(c, seed):
    """Queries, keys, values and gates as one product writes them, side by side in its rows."""
    T, B, H, dk, dv = c.get("T", 1), c["B"], c["H"], c["dk"], c["dv"]
    s = dict(kind=c["kind"], c=c, lam=_decays(seed, H), done=None, lens=None,
             proj=_normal(seed, 4, (T, B, H * (2 * dk + dv + 2)), _torch(c)),
             h0=_normal(seed, 5, (B, H, dk, dv), scale=0.3))
    if c["kind"] == "step":
        s["done"] = (torch.rand(T, B, generator=_gen(seed, 6), device=DEV) < 1 / 256).byte()
        return s
    if c["ends"]:
        s["done"] = (torch.rand(T, B, generator=_gen(seed, 6), device=DEV) < c["ends"]).byte()
    s["lens"] = _lens(c, seed)
    if c["kind"] == "train":
        s["dy"] = _normal(seed, 8, (T, B, H, dv), _torch(c))
        s["dh_last"] = _normal(seed, 9, (B, H, dk, dv), scale=0.3)
    return s


def _norm_inputs(c, seed):
    """The residual stream, a block's output, and its gate as a part of a product's rows."""
    M, D = c["rows"], c["D"]
    s = dict(kind=c["kind"], c=c, x=_normal(seed, 2, (M, D), _torch(c), 2.0),
             y=_normal(seed, 3, (M, D), _torch(c), 0.5),
             z=_normal(seed, 4, (M, D + 8), _torch(c))[:, 8:])
    s["w_post"] = 1.0 + _normal(seed, 5, (D,), scale=0.2)
    s["w_pre"] = 1.0 + _normal(seed, 6, (D,), scale=0.2)
    s["scale"] = 0.3 + _normal(seed, 7, (D,), scale=0.1)
    if c["kind"] == "normgrad":
        s["dx_out"] = _normal(seed, 8, (M, D), _torch(c))
        s["dn"] = _normal(seed, 9, (M, D), _torch(c))
    return s


def _loss_inputs(c, seed):
    """A policy some updates after the rollout: means that moved a little, actions drawn around the
    old ones, standardised advantages."""
    T, B, n = c["T"], c["B"], c["n"]
    ref_std = -1.0 + _normal(seed, 2, (n,), scale=0.1)
    mu_ref = _normal(seed, 3, (T, B, n), scale=0.5)
    z = _normal(seed, 4, (T, B, n))
    action = mu_ref + torch.exp(ref_std) * z
    logp = (-0.5 * z.double().square() - ref_std.double()).sum(2) - 0.5 * n * math.log(2 * math.pi)
    move = 0.3 / math.sqrt(n)
    mu = mu_ref + _normal(seed, 5, (T, B, n), scale=1.0).mul_(move * torch.exp(ref_std))
    return dict(kind="loss", c=c, mu=mu.to(_torch(c)), action=action, mu_ref=mu_ref,
                logp=logp.float(), adv=_normal(seed, 6, (T, B)),
                log_std=ref_std + _normal(seed, 8, (n,), scale=0.1 * move),
                log_std_ref=ref_std, lens=_lens(c, seed), clip=(0.2, 0.28), kl=0.05, ent=0.02)


def _inputs(c, seed):
    if c["kind"] == "loss":
        return _loss_inputs(c, seed)
    return (_norm_inputs if "norm" in c["kind"] else _delta_inputs)(c, seed)


def prepare(c, seed):
    s = _inputs(c, seed)
    if own:
        _buffers(s)                         # descriptors, outputs, workspaces
    return s


def _parts(p, c):
    """Views of a product's rows: q, k [..][H][dk], v [..][H][dv], r, b [..][H]."""
    H, dk, dv = c["H"], c["dk"], c["dv"]
    at = [0, H * dk, 2 * H * dk, H * (2 * dk + dv), H * (2 * dk + dv + 1), H * (2 * dk + dv + 2)]
    q, k, v, r, b = (p[..., i:j] for i, j in zip(at, at[1:]))
    return (q.unflatten(-1, (H, dk)), k.unflatten(-1, (H, dk)), v.unflatten(-1, (H, dv)), r, b)


# --------------------------------------------------------------------------
# the plain forms: the delta rule in chunks
# --------------------------------------------------------------------------

CHUNK = 32


def _sigmoid(x):
    return 1.0 / (1.0 + torch.exp(-x))


def _softplus(x):
    return torch.clamp(x, min=0.0) + torch.log1p(torch.exp(-torch.abs(x)))


def _chunk(s, t0):
    """One chunk with heads as a batch [B H][C][.], in fp32: unit queries and keys, the products'
    triangles with their decays, and the inverse that turns targets into writes.  Steps past a
    sequence's end neither write nor decay; decays stop at an episode's end."""
    c = s["c"]
    T, B, H = c.get("T", 1), c["B"], c["H"]
    t1 = min(t0 + CHUNK, T)
    n = t1 - t0
    q, k, v, r, b = (p[t0:t1].movedim(0, 2).reshape(B * H, n, -1).float()
                     for p in _parts(s["proj"], c))
    valid = torch.ones(n, B, dtype=torch.bool, device=DEV)
    if s["lens"] is not None:
        valid = torch.arange(t0, t1, device=DEV)[:, None] < s["lens"][None]
    ends = torch.zeros(n, B, device=DEV)
    if s["done"] is not None:
        ends = (s["done"][t0:t1] != 0).float() * valid
    spread = lambda m: m.t()[:, None].expand(B, H, n).reshape(B * H, n)  # noqa: E731
    valid, ends = spread(valid)[..., None], spread(ends)
    rate = (-8.0 * _softplus(s["lam"].double()))[None].expand(B, H).reshape(-1, 1, 1)
    o = dict(n=n, t0=t0, t1=t1, valid=valid, rho=_sigmoid(r))
    o["g"] = torch.where(valid, rate * _sigmoid(r.double()), 0.0)
    o["beta"] = torch.where(valid, _sigmoid(b), 0.0)
    o["rq"] = 1.0 / torch.sqrt(q.square().sum(-1, keepdim=True) + EPS)
    o["rk"] = 1.0 / torch.sqrt(k.square().sum(-1, keepdim=True) + EPS)
    o["q"] = torch.where(valid, q * o["rq"], 0.0)
    o["k"] = torch.where(valid, k * o["rk"], 0.0)
    o["v"] = torch.where(valid, v, 0.0)
    after = torch.cumsum(ends, 1)
    part = (after - ends)[..., None]                    # the episode, counted within the chunk
    o["same"] = part == part.transpose(1, 2)
    o["first"], o["last"] = part == 0, part == after[:, -1:, None]
    total = torch.cumsum(o["g"], 1)
    low = torch.ones(n, n, device=DEV).tril()
    o["low"] = low
    fade = torch.exp(torch.where(o["same"] & (low > 0), total - total.transpose(1, 2),
                                 -torch.inf)).float()
    o["fade"] = fade
    o["fade_in"] = torch.exp(torch.where(o["first"], total, -torch.inf)).float()
    o["fade_out"] = torch.exp(torch.where(o["last"], total[:, -1:] - total, -torch.inf)).float()
    o["keep"] = torch.where(after[:, -1:, None] == 0, torch.exp(total[:, -1:]).float(), 0.0)
    kt = o["k"].transpose(1, 2).contiguous()
    o["P"] = (o["q"] @ kt) * fade
    o["KK"] = (o["k"] @ kt) * (fade * low.tril(-1))
    A = o["beta"] * o["KK"]
    inv = torch.eye(n, device=DEV).expand(B * H, n, n)  # blocks of 1, 2, 4 .. on the diagonal
    at = torch.arange(n, device=DEV)
    w = 1
    while w < n:
        off = (at[:, None] // (2 * w) == at[None] // (2 * w)) & (at[:, None] // w != at[None] // w)
        inv = inv - inv @ (A * off) @ inv
        w *= 2
    o["inv"] = inv
    return o


def _writes(o, S):
    R = o["beta"] * (o["v"] - o["fade_in"] * (o["k"] @ S))
    return o["inv"] @ R


def _next(o, S, U):
    # (the last step may end the episode: then nothing goes on)
    return o["keep"] * S + (o["k"] * o["fade_out"]).transpose(1, 2).contiguous() @ U


def _delta_forward(s):
    c = s["c"]
    T, B, H, dk, dv = c.get("T", 1), c["B"], c["H"], c["dk"], c["dv"]
    S = s["h0"].reshape(B * H, dk, dv)
    y = torch.zeros(T, B, H, dv, dtype=_torch(c), device=DEV)
    starts = []
    for t0 in range(0, T, CHUNK):
        o = _chunk(s, t0)
        U = _writes(o, S)
        out = o["fade_in"] * (o["q"] @ S) + o["P"] @ U
        y[o["t0"]:o["t1"]] = out.view(B, H, o["n"], dv).movedim(2, 0).to(y.dtype)
        starts.append(S if c["kind"] == "train" else None)
        S = _next(o, S, U)
    return y, S.view(B, H, dk, dv), starts


def _unit_grad(d, x, r):
    """The gradient through x r, r = 1/length, of unit rows x."""
    return r * (d - x * (x * d).sum(-1, keepdim=True))


def _delta_backward(s, starts):
    c = s["c"]
    T, B, H, dk, dv = c["T"], c["B"], c["H"], c["dk"], c["dv"]
    G = s["dh_last"].reshape(B * H, dk, dv)
    dproj = torch.zeros_like(s["proj"])
    into = _parts(dproj, c)
    dlam = torch.zeros(B, H, dtype=torch.float64, device=DEV)
    rate = (-8.0 * _softplus(s["lam"]))[None].expand(B, H).reshape(-1, 1, 1)
    turn = lambda m: m.transpose(1, 2).contiguous()  # noqa: E731
    for t0 in reversed(range(0, T, CHUNK)):
        o, S = _chunk(s, t0), starts[t0 // CHUNK]
        n = o["n"]
        dy = s["dy"][o["t0"]:o["t1"]].movedim(0, 2).reshape(B * H, n, dv).float()
        dy = torch.where(o["valid"], dy, 0.0)
        U = _writes(o, S)
        end = (G * _next(o, S, U)).sum((1, 2)).double()[:, None, None]
        dU = turn(o["P"]) @ dy + o["fade_out"] * (o["k"] @ G)
        dR = turn(o["inv"]) @ dU
        St, Gt, Ut = turn(S), turn(G), turn(U)
        dP = (dy @ Ut) * o["fade"]
        E = -(dR @ Ut) * o["beta"] * (o["fade"] * o["low"].tril(-1))
        dq = o["fade_in"] * (dy @ St) + dP @ o["k"]
        dk_ = (-o["beta"] * o["fade_in"] * (dR @ St) + o["fade_out"] * (U @ Gt) +
               turn(dP) @ o["q"] + (E + turn(E)) @ o["k"])
        rows = (dR * U).sum(-1, keepdim=True)
        # what multiplies the state at a step: all that reads or becomes it until the episode ends
        x = ((o["q"] * dq).sum(-1, keepdim=True).double() +
             (o["k"] * dk_).sum(-1, keepdim=True).double() - 2.0 * rows.double())
        later = (o["same"] & (o["low"].t() > 0)).double()
        dg = later @ x + torch.where(o["last"], end, 0.0)
        w = torch.where(o["valid"], dg * o["g"], 0.0).float()
        grads = (_unit_grad(dq, o["q"], o["rq"]), _unit_grad(dk_, o["k"], o["rk"]),
                 o["beta"] * dR, w * (1.0 - o["rho"]), rows * (1.0 - o["beta"]))
        for d, m in zip(into, grads):
            m = torch.where(o["valid"], m, 0.0)
            if d.dim() == 3:
                d[o["t0"]:o["t1"]] = m.view(B, H, n).movedim(2, 0).to(d.dtype)
            else:
                d[o["t0"]:o["t1"]] = m.view(B, H, n, -1).movedim(2, 0).to(d.dtype)
        dlam += w.double().sum((1, 2)).view(B, H)
        G = (o["keep"] * G + turn(o["q"] * o["fade_in"]) @ dy -
             turn(o["k"] * (o["beta"] * o["fade_in"])) @ dR)
    lam = s["lam"].double()
    dlam = dlam.sum(0) * (_sigmoid(lam) / _softplus(lam))
    return dproj, dlam.float(), G.view(B, H, dk, dv)


# --------------------------------------------------------------------------
# the plain forms: norms, loss
# --------------------------------------------------------------------------

def _norm_forward(s):
    c = s["c"]
    M, D, G = c["rows"], c["D"], c["groups"]
    x, y, z = s["x"].float(), s["y"].float(), s["z"].float()
    y = y.view(M, G, D // G)
    ry = 1.0 / torch.sqrt(y.square().mean(2, keepdim=True) + EPS)
    yn = (y * ry).view(M, D)
    gate = _sigmoid(z)
    f = yn * s["w_post"] * (z * gate)
    X = x + s["scale"] * f
    rx = 1.0 / torch.sqrt(X.square().mean(1, keepdim=True) + EPS)
    return X, rx, yn, ry, z, gate, f


def _norm_backward(s, kept):
    c = s["c"]
    M, D, G = c["rows"], c["D"], c["groups"]
    X, rx, yn, ry, z, gate, f = kept
    dn = s["dn"].float()
    xn = X * rx
    t = dn * s["w_pre"]
    dw_pre = (dn * xn).double().sum(0)
    dX = s["dx_out"].float() + rx * (t - xn * (t * xn).mean(1, keepdim=True))
    dscale = (dX * f).double().sum(0)
    df = dX * s["scale"]
    dw_post = (df * yn * (z * gate)).double().sum(0)
    dz = df * yn * s["w_post"] * (gate * (1.0 + z * (1.0 - gate)))
    dyn = (df * s["w_post"] * (z * gate)).view(M, G, D // G)
    yg = yn.view(M, G, D // G)
    dy = (ry * (dyn - yg * (dyn * yg).mean(2, keepdim=True))).view(M, D)
    to = lambda m: m.to(_torch(c))  # noqa: E731
    return dict(dx=to(dX), dy=to(dy), dz=to(dz), dw_post=dw_post.float(), dscale=dscale.float(),
                dw_pre=dw_pre.float())


def _loss(s):
    """In 64 bits up to the ratio: a rounding would put some of many rows on the other side of the
    clip."""
    c = s["c"]
    T, B, n = c["T"], c["B"], c["n"]
    lo, hi = s["clip"]
    ls, lr = s["log_std"].double(), s["log_std_ref"].double()
    inv = torch.exp(-ls)
    mu = s["mu"].double()
    z = (s["action"].double() - mu) * inv
    logp = (-0.5 * z.square()).sum(2) - ls.sum() - 0.5 * n * math.log(2 * math.pi)
    ratio = torch.exp(logp - s["logp"].double())
    A = s["adv"].double()
    clipped = torch.clamp(ratio, 1.0 - lo, 1.0 + hi)
    valid = torch.ones(T, B, dtype=torch.bool, device=DEV)
    if s["lens"] is not None:
        valid = torch.arange(T, device=DEV)[:, None] < s["lens"][None]
    N = valid.double().sum()
    share = torch.where(N > 0, 1.0 / torch.clamp(N, min=1.0), 0.0)
    mean = lambda m: torch.where(valid, m, 0.0).sum() * share  # noqa: E731
    off = (mu - s["mu_ref"].double()) * inv
    spread = torch.exp(2.0 * (lr - ls))
    kl = (ls - lr - 0.5 + 0.5 * spread + 0.5 * off.square()).sum(2)
    surrogate = torch.minimum(ratio * A, clipped * A)
    entropy = (ls + 0.5 * (1.0 + math.log(2 * math.pi))).sum()
    policy, KL = -mean(surrogate), mean(kl)
    out = mean(((ratio < 1.0 - lo) | (ratio > 1.0 + hi)).double())
    total = policy + s["kl"] * KL - s["ent"] * entropy
    w = torch.where(valid & (ratio * A <= clipped * A), -ratio * A * share, 0.0)[..., None]
    k = torch.where(valid, s["kl"] * share, 0.0)[..., None]
    dmu = torch.where(valid[..., None], w * z * inv + k * off * inv, 0.0)
    dls = torch.where(valid[..., None], w * (z.square() - 1.0) +
                      k * (1.0 - spread - off.square()), 0.0).sum((0, 1)) - s["ent"]
    return dict(stats=torch.stack([total, policy, KL, entropy, out, N]), dmu=dmu.to(_torch(c)),
                dlog_std=dls.float())


def _plain(s):
    kind, c = s["kind"], s["c"]
    if kind in ("step", "scan"):
        y, h, _ = _delta_forward(s)
        return dict(y=y[0] if kind == "step" else y, h_last=h)
    if kind == "train":
        y, h, starts = _delta_forward(s)
        dproj, dlam, dh0 = _delta_backward(s, starts)
        return dict(y=y, h_last=h, dproj=dproj, dlam=dlam, dh0=dh0)
    if kind == "loss":
        return _loss(s)
    kept = _norm_forward(s)
    out = dict(x_out=kept[0].to(_torch(c)), n=(kept[0] * kept[1] * s["w_pre"]).to(_torch(c)))
    if kind == "normgrad":
        out.update(_norm_backward(s, kept))
    return out


# --------------------------------------------------------------------------
# the framework's operators
# --------------------------------------------------------------------------

def _buffers(s):
    """What a program keeps between calls: descriptors, outputs and workspaces."""
    from paper_2111_05188_amd import tp
    kind, c = s["kind"], s["c"]
    f32 = torch.float32
    new = lambda *shape, dtype=_torch(c): torch.empty(shape, dtype=dtype, device=DEV)  # noqa: E731
    if kind == "step":
        B, H, dk, dv = c["B"], c["H"], c["dk"], c["dv"]
        s["y"], s["h_next"] = new(B, H, dv), new(B, H, dk, dv, dtype=f32)
    elif kind in ("scan", "train"):
        T, B, H, dk, dv = c["T"], c["B"], c["H"], c["dk"], c["dv"]
        s["dc"] = dc = tp.DeltaT(s["lam"], T, B, dk, dv, _torch(c), done=s["done"], lens=s["lens"])
        s["work"], s["y"] = dc.workspace(), new(T, B, H, dv)
        s["h_last"] = new(B, H, dk, dv, dtype=f32)
        if kind == "train":
            s["saved"], s["dproj"] = dc.saved(), torch.empty_like(s["proj"])
            s["dlam"], s["dh0"] = new(H, dtype=f32), new(B, H, dk, dv, dtype=f32)
    elif kind == "loss":
        s["pc"] = tp.PolicyT(s["log_std"], c["T"], c["B"], _torch(c), clip=s["clip"],
                             kl_coef=s["kl"], ent_coef=s["ent"], log_std_ref=s["log_std_ref"],
                             lens=s["lens"])
        s["work"], s["dmu"] = s["pc"].workspace(), torch.empty_like(s["mu"])
        s["dlog_std"], s["stats"] = new(c["n"], dtype=f32), new(6, dtype=torch.float64)
    else:
        M, D = c["rows"], c["D"]
        s["nc"] = tp.NormT(M, D, _torch(c), w_pre=s["w_pre"], w_post=s["w_post"],
                           scale=s["scale"], groups=c["groups"], eps=EPS)
        s["x_out"], s["n"] = new(M, D), new(M, D)
        if kind == "normgrad":
            s["work"] = s["nc"].workspace()
            for k in ("dx", "dy", "dz"):
                s[k] = new(M, D)
            for k in ("dw_post", "dscale", "dw_pre"):
                s[k] = new(D, dtype=f32)


def _run(s):
    from paper_2111_05188_amd import tp
    kind, c = s["kind"], s["c"]
    if kind == "step":
        tp.delta_step(*_parts(s["proj"][0], c), s["lam"], s["h0"], s["h_next"], s["y"],
                      done=s["done"][0])
        return dict(y=s["y"], h_last=s["h_next"])
    if kind in ("scan", "train"):
        parts = _parts(s["proj"], c)
        tp.delta_forward(s["dc"], *parts, s["y"], s["work"], h0=s["h0"], h_last=s["h_last"],
                         saved=s.get("saved"))
        if kind == "scan":
            return dict(y=s["y"], h_last=s["h_last"])
        tp.delta_backward(s["dc"], *parts, s["saved"], s["dy"], *_parts(s["dproj"], c), s["dlam"],
                          s["work"], dh_last=s["dh_last"], dh0=s["dh0"])
        return {k: s[k] for k in ("y", "h_last", "dproj", "dlam", "dh0")}
    if kind == "loss":
        tp.policy_loss(s["pc"], s["mu"], s["action"], s["logp"], s["adv"], s["work"], s["stats"],
                       s["dmu"], s["dlog_std"], mu_ref=s["mu_ref"])
        return {k: s[k] for k in ("stats", "dmu", "dlog_std")}
    tp.norm_forward(s["nc"], s["x"], s["y"], s["z"], s["x_out"], s["n"])
    out = dict(x_out=s["x_out"], n=s["n"])
    if kind == "normgrad":
        tp.norm_backward(s["nc"], s["x"], s["y"], s["z"], s["dx_out"], s["dn"], s["dx"], s["dy"],
                         s["dz"], s["dw_post"], s["dscale"], s["dw_pre"], s["work"])
        out.update((k, s[k]) for k in ("dx", "dy", "dz", "dw_post", "dscale", "dw_pre"))
    return out


def run(s):
    return _run(s) if own else _plain(s)


# --------------------------------------------------------------------------
# the definitions in 64 bits
# --------------------------------------------------------------------------

def _exact_step(p, lam, S):
    """One step of all heads, and what its gradient needs: p are a step's q, k, v, r, b."""
    q, k, v, r, b = p
    rho, beta = torch.sigmoid(r), torch.sigmoid(b)
    g = -8.0 * torch.nn.functional.softplus(lam) * rho
    q = q / torch.sqrt(q.square().sum(-1, keepdim=True) + EPS)
    k = k / torch.sqrt(k.square().sum(-1, keepdim=True) + EPS)
    S1 = torch.exp(g)[..., None, None] * S
    e = v - (S1 * k[..., None]).sum(-2)
    u = beta[..., None] * e
    S2 = S1 + k[..., None] * u[..., None, :]
    return S2, (S2 * q[..., None]).sum(-2), (rho, beta, g, q, k, S1, e, u)


def _exact_gates(s, t, S):
    """Which sequences are in step t, and which end an episode with it."""
    live = torch.ones(S.shape[0], dtype=torch.bool, device=DEV)
    if s["lens"] is not None:
        live = t < s["lens"]
    ends = live & (s["done"][t] != 0) if s["done"] is not None else torch.zeros_like(live)
    return live[:, None, None], live[:, None, None, None], ends[:, None, None, None]


def _exact_forward(s, t0, t1, S, keep=None):
    ys = []
    lam = s["lam"].double()
    for t in range(t0, t1):
        live, live4, ends = _exact_gates(s, t, S)
        if keep is not None:
            keep.append(S)
        p = [m.double() for m in _parts(s["proj"][t], s["c"])]
        new, y, _ = _exact_step(p, lam, S)
        ys.append(torch.where(live, y, 0.0))
        S = torch.where(ends, 0.0, torch.where(live4, new, S))
    return ys, S


def _exact_delta(s):
    c = s["c"]
    T, B, H, dk, dv = c.get("T", 1), c["B"], c["H"], c["dk"], c["dv"]
    S, lam = s["h0"].double(), s["lam"].double()
    if c["kind"] != "train":
        ys, S = _exact_forward(s, 0, T, S)
        return dict(y=ys[0] if c["kind"] == "step" else torch.stack(ys), h_last=S)
    part = max(1, math.isqrt(T))                        # the states again from every part's first
    marks, ys = [], []
    for t0 in range(0, T, part):
        marks.append(S)
        more, S = _exact_forward(s, t0, min(T, t0 + part), S)
        ys += more
    dproj = torch.zeros_like(s["proj"], dtype=torch.float64)
    into = _parts(dproj, c)
    dlam = torch.zeros(H, dtype=torch.float64, device=DEV)
    G = s["dh_last"].double()
    for i in reversed(range(len(marks))):
        before = []
        t0, t1 = i * part, min(T, (i + 1) * part)
        _exact_forward(s, t0, t1, marks[i], before)
        for t in reversed(range(t0, t1)):
            live, live4, ends = _exact_gates(s, t, S)
            p = [m.double() for m in _parts(s["proj"][t], c)]
            S2, _, (rho, beta, g, q, k, S1, e, u) = _exact_step(p, lam, before[t - t0])
            dy = s["dy"][t].double()
            D2 = torch.where(ends, 0.0, G) + q[..., None] * dy[..., None, :]
            dq = (S2 * dy[..., None, :]).sum(-1)
            du = (D2 * k[..., None]).sum(-2)
            dk_ = (D2 * u[..., None, :]).sum(-1)
            dbeta = (du * e).sum(-1)
            de = beta[..., None] * du
            D1 = D2 - k[..., None] * de[..., None, :]
            dk_ = dk_ - (S1 * de[..., None, :]).sum(-1)
            dg = (D1 * S1).sum((-2, -1))
            through = []                                # x / sqrt(x.x + eps)
            for x, unit, d in ((p[0], q, dq), (p[1], k, dk_)):
                length = torch.sqrt(x.square().sum(-1, keepdim=True) + EPS)
                through.append((d - unit * (unit * d).sum(-1, keepdim=True)) / length)
            on = live[..., 0]
            dlam += torch.where(on, dg * g, 0.0).sum(0)
            for d, m in zip(into, (*through, de, dg * g * (1.0 - rho),
                                   dbeta * beta * (1.0 - beta))):
                d[t] = torch.where(live if m.dim() == 3 else on, m, 0.0)
            G = torch.where(live4, torch.exp(g)[..., None, None] * D1, G)
    dlam = dlam * torch.sigmoid(lam) / torch.nn.functional.softplus(lam)
    return dict(y=torch.stack(ys), h_last=S, dproj=dproj, dlam=dlam, dh0=G)


def _exact_norm(s):
    """Gradients by differentiating the definition."""
    c, train = s["c"], s["c"]["kind"] == "normgrad"
    M, D, G = c["rows"], c["D"], c["groups"]
    names = ("x", "y", "z", "w_post", "scale", "w_pre")
    part = max(1, 100_000_000 // D)
    rows, sums = [], {}
    for m in range(0, M, part):
        e = slice(m, m + part)
        p = {k: (s[k][e] if k in "xyz" else s[k]).double().requires_grad_(train) for k in names}
        with torch.set_grad_enabled(train):
            y = p["y"].unflatten(1, (G, D // G))
            y = (y / torch.sqrt(y.pow(2).mean(2, keepdim=True) + EPS)).flatten(1)
            x = p["x"] + p["scale"] * (p["w_post"] * y * p["z"] * torch.sigmoid(p["z"]))
            n = p["w_pre"] * x / torch.sqrt(x.pow(2).mean(1, keepdim=True) + EPS)
            if train:
                ((x * s["dx_out"][e].double()).sum() + (n * s["dn"][e].double()).sum()).backward()
        out = dict(x_out=x.detach(), n=n.detach())
        if train:
            out.update({"d" + k: p[k].grad for k in "xyz"})
            for k in names[3:]:
                sums["d" + k] = sums.get("d" + k, 0.0) + p[k].grad
        rows.append(out)
    return {**{k: torch.cat([r[k] for r in rows]) for k in rows[0]}, **sums}


def _exact_loss(s):
    """Gradients by differentiating the definition, over the rows that the sequences have."""
    c = s["c"]
    mu, ls = s["mu"].double().requires_grad_(), s["log_std"].double().requires_grad_()
    old, lr = torch.distributions.Normal, s["log_std_ref"].double()
    on = torch.ones(c["T"], c["B"], dtype=torch.bool, device=DEV)
    if s["lens"] is not None:
        on = torch.arange(c["T"], device=DEV)[:, None] < s["lens"][None]
    N = int(on.sum())
    new = old(mu[on], ls.exp())
    entropy = old(torch.zeros_like(ls), ls.exp()).entropy().sum()
    policy = KL = out = torch.zeros((), dtype=torch.float64, device=DEV)
    if N:
        ratio = (new.log_prob(s["action"][on].double()).sum(1) - s["logp"][on].double()).exp()
        A, (lo, hi) = s["adv"][on].double(), s["clip"]
        policy = -torch.minimum(ratio * A, ratio.clamp(1.0 - lo, 1.0 + hi) * A).mean()
        KL = torch.distributions.kl_divergence(old(s["mu_ref"][on].double(), lr.exp()),
                                               new).sum(1).mean()
        out = ((ratio < 1.0 - lo) | (ratio > 1.0 + hi)).double().mean()
    total = policy + s["kl"] * KL - s["ent"] * entropy
    total.backward()
    dmu = mu.grad if mu.grad is not None else torch.zeros_like(mu)
    stats = torch.stack([total, policy, KL, entropy, out, out.new_tensor(float(N))]).detach()
    return dict(stats=stats, dmu=dmu, dlog_std=ls.grad)


def exact(c, seed):
    s = _inputs(c, seed)
    if c["kind"] == "loss":
        return _exact_loss(s)
    return (_exact_norm if "norm" in c["kind"] else _exact_delta)(s)
