"""A policy made of residual blocks with a matrix memory, and its training step on what a rollout
stores.

  x_0 = obs E^T,  n_0 = norm(x_0)                    tp.mx4_linear, tp.norm_forward
  block i:  [q k v z r b] = n_i W_i^T                tp.mx4_linear
            y = delta rule(q, k, v, r, b)            tp.delta_forward, one bar: tp.delta_step
            x_{i+1} = x_i + scale norm(y) silu(z),   tp.norm_forward
            n_{i+1} = norm(x_{i+1})
  mu = n O^T + bias                                  tp.mx4_linear

and back: tp.policy_loss gives mu's gradient (clipped ratio, entropy, KL to the policy that acted, whose
means a rollout stores as mu_tap), tp.norm_backward and tp.delta_backward take it through the blocks.
The matrices' fp32 masters go to 4 bits for every product, forward and back, as memory.MemoryLayer's
do; the rounding counts as the identity in the gradients.  Everything runs on torch's current stream and
every call takes buffers of its own from torch; forward, loss and gradients of a batch belong on one
stream, and the forward's observations, done and lens stay as they are until its gradients are there.

Plumbing only (buffers and the order of calls); `python -m paper_2111_05188_amd.policy` trains a policy
to trade on the mean of the last bars.
"""

from __future__ import annotations

import math

import torch

from . import tp


class Matrix:
    """A matrix W [N][K] fp32 and its 4-bit forms for the product, the gradient of its input and
    (over the rows of a call) its own."""

    def __init__(self, W: torch.Tensor):
        self.W = W
        self.refresh()

    def refresh(self):
        self.w4, self.wt4 = tp.mx4_quantize(self.W), tp.mx4_quantize(self.W.t())

    def forward(self, x, bias=None):
        y = torch.empty(x.shape[0], self.W.shape[0], dtype=x.dtype, device=x.device)
        tp.mx4_linear(x, self.w4, y, bias=bias)
        return y

    def gradients(self, x, dy, dx=True):
        """dW [N][K] and (if wanted) dx of y = x W^T."""
        dW = torch.empty_like(self.W)
        tp.mx4_matmul(tp.mx4_quantize(dy.t()), tp.mx4_quantize(x.t()), dW)
        if not dx:
            return dW, None
        out = torch.empty(x.shape[0], self.W.shape[1], dtype=x.dtype, device=x.device)
        tp.mx4_linear(dy, self.wt4, out)
        return dW, out


class Block:
    """H heads of d channels on a residual stream of H d."""

    def __init__(self, H: int, d: int, g: torch.Generator, device):
        self.H, self.d, D = H, d, H * d
        self.m = Matrix(torch.randn(H * (4 * d + 2), D, generator=g, device=device) * D ** -0.5)
        a = 1.0 - 10.0 ** -torch.linspace(1.0, 3.0, H, device=device)       # memories of 10 to 1,000 bars
        self.lam = torch.log(torch.expm1(-torch.log(a) / 4.0))
        self.w_pre, self.w_post = torch.ones(D, device=device), torch.ones(D, device=device)
        self.scale = torch.full((D,), 0.5, device=device)

    def parts(self, p):
        """q, k, v, r, b with heads as an axis of their own, and z, of a product's rows."""
        H, d, D = self.H, self.d, self.H * self.d
        q, k, v, z = (p[..., i * D:(i + 1) * D] for i in range(4))
        head = lambda t: t.unflatten(-1, (H, d))  # noqa: E731
        return (head(q), head(k), head(v), p[..., 4 * D:4 * D + H], p[..., 4 * D + H:]), z

    def parameters(self):
        return dict(W=self.m.W, lam=self.lam, w_pre=self.w_pre, w_post=self.w_post, scale=self.scale)


class MatrixPolicy:
    """Means of n actions from observations of S features; log_std [n] is a parameter of its own."""

    def __init__(self, S: int, n: int, H: int = 4, d: int = 32, blocks: int = 2, dtype=torch.bfloat16,
                 seed: int = 0, device="cuda"):
        g = torch.Generator(device=device).manual_seed(seed)
        self.S, self.n, self.D, self.dtype = S, n, H * d, dtype
        self.embed = Matrix(torch.randn(self.D, S, generator=g, device=device) * S ** -0.5)
        self.blocks = [Block(H, d, g, device) for _ in range(blocks)]
        self.w_out = torch.ones(self.D, device=device)
        self.head = Matrix(torch.randn(n, self.D, generator=g, device=device) * 0.1 * self.D ** -0.5)
        self.bias = torch.zeros(n, device=device)
        self.log_std = torch.full((n,), -1.0, device=device)

    def parameters(self):
        """Name -> fp32 tensor, in the order and with the names of gradients()."""
        out = dict(embed=self.embed.W)
        for i, b in enumerate(self.blocks):
            out.update({f"{i}.{k}": v for k, v in b.parameters().items()})
        out.update(w_out=self.w_out, head=self.head.W, bias=self.bias, log_std=self.log_std)
        return out

    def refresh(self):
        """The 4-bit forms again, after an optimiser has changed the parameters."""
        for m in (self.embed, self.head, *(b.m for b in self.blocks)):
            m.refresh()

    def _norm(self, i: int, rows: int):
        """The norms between block i - 1 and block i (or the head)."""
        after = self.blocks[i - 1] if i else None
        return tp.NormT(rows, self.D, self.dtype,
                        w_pre=self.blocks[i].w_pre if i < len(self.blocks) else self.w_out,
                        w_post=after and after.w_post, scale=after and after.scale,
                        groups=after.H if after else 1)

    def states(self, B: int):
        """First states of B sequences: zeros."""
        return [torch.zeros(B, b.H, b.d, b.d, device=self.w_out.device) for b in self.blocks]

    def forward(self, obs, done=None, lens=None, states=None):
        """Means [T][B][n] of stored observations [T][B][ld] (ld >= S); `states`, those before the
        first bar, become those after the last.  Keeps what gradients() reads."""
        T, B, ld = obs.shape
        M = T * B
        rows = obs.reshape(M, ld)
        if lens is not None:            # what lies past a sequence shares blocks with what counts
            past = torch.arange(T, device=obs.device)[:, None] >= lens
            rows = rows.masked_fill(past.view(-1, 1), 0.0)
        new = lambda *s: torch.empty(*s, dtype=self.dtype, device=obs.device)  # noqa: E731
        self.T, self.B, self.rows = T, B, rows[:, :self.S]
        x, n = self.embed.forward(self.rows), new(M, self.D)
        tp.norm_forward(self._norm(0, M), x, None, None, None, n)
        self.kept = []
        for i, b in enumerate(self.blocks):
            dc = tp.DeltaT(b.lam, T, B, b.d, b.d, self.dtype, done=done, lens=lens)
            p, y, saved = b.m.forward(n), new(T, B, b.H, b.d), dc.saved()
            qkvrb, z = b.parts(p.view(T, B, -1))
            h = None if states is None else states[i]
            tp.delta_forward(dc, *qkvrb, y, dc.workspace(), h0=h, h_last=h, saved=saved)
            x_out, n_out = new(M, self.D), new(M, self.D)
            tp.norm_forward(self._norm(i + 1, M), x, y.view(M, -1), z.view(M, -1), x_out, n_out)
            self.kept.append((dc, x, n, p, y, saved))
            x, n = x_out, n_out
        self.last = n
        return self.head.forward(n, self.bias).view(T, B, self.n)

    def loss(self, mu, action, logp, adv, mu_ref=None, log_std_ref=None, lens=None, clip=0.25,
             kl_coef=0.0, ent_coef=0.02):
        """stats [6], dmu and dlog_std of tp.policy_loss; action, logp, adv, mu_ref as stored."""
        pc = tp.PolicyT(self.log_std, self.T, self.B, self.dtype, clip=clip, kl_coef=kl_coef,
                        ent_coef=ent_coef, log_std_ref=log_std_ref, lens=lens)
        stats = torch.empty(6, dtype=torch.float64, device=mu.device)
        dmu, dlog_std = torch.empty_like(mu), torch.empty_like(self.log_std)
        tp.policy_loss(pc, mu, action, logp, adv, pc.workspace(), stats, dmu, dlog_std, mu_ref=mu_ref)
        return stats, dmu, dlog_std

    def gradients(self, dmu, dlog_std):
        """Gradients of parameters() from those of the last forward's means (first states' are not
        kept)."""
        M = self.T * self.B
        dmu = dmu.view(M, self.n)
        out = dict(log_std=dlog_std, bias=dmu.float().sum(0))
        out["head"], dn = self.head.gradients(self.last, dmu)
        dx, f32 = None, dict(dtype=torch.float32, device=dmu.device)
        for i in reversed(range(len(self.blocks))):
            b, (dc, x, n, p, y, saved) = self.blocks[i], self.kept[i]
            _, z = b.parts(p)
            dp, dy, dx_in = torch.empty_like(p), torch.empty_like(y), torch.empty_like(x)
            dqkvrb, dz = b.parts(dp.view(self.T, self.B, -1))
            dw_post, dscale, dw_next, dlam = (torch.empty(k, **f32) for k in (self.D, self.D, self.D, b.H))
            nc = self._norm(i + 1, M)
            tp.norm_backward(nc, x, y.view(M, -1), z, dx, dn, dx_in, dy.view(M, -1), dz.view(M, -1),
                             dw_post, dscale, dw_next, nc.workspace())
            tp.delta_backward(dc, *b.parts(p.view(self.T, self.B, -1))[0], saved, dy, *dqkvrb, dlam,
                              dc.workspace())
            dW, dn = b.m.gradients(n, dp)
            out.update({f"{i}.W": dW, f"{i}.lam": dlam, f"{i}.w_post": dw_post, f"{i}.scale": dscale})
            out["w_out" if i + 1 == len(self.blocks) else f"{i + 1}.w_pre"] = dw_next
            dx = dx_in
        x, nc = self.kept[0][1], self._norm(0, M)
        dx_in, dw_pre = torch.empty_like(x), torch.empty(self.D, **f32)
        tp.norm_backward(nc, x, None, None, dx, dn, dx_in, None, None, None, None, dw_pre, nc.workspace())
        out["0.w_pre"] = dw_pre
        out["embed"], _ = self.embed.gradients(self.rows, dx_in, dx=False)
        return {k: out[k] for k in self.parameters()}

    def step(self, obs, states, done=None):
        """Means [B][n] of one bar's observations [B][ld]; the states move on in place."""
        B = obs.shape[0]
        new = lambda: torch.empty(B, self.D, dtype=self.dtype, device=obs.device)  # noqa: E731
        x, n = self.embed.forward(obs[:, :self.S]), new()
        tp.norm_forward(self._norm(0, B), x, None, None, None, n)
        for i, b in enumerate(self.blocks):
            qkvrb, z = b.parts(b.m.forward(n))
            y, n_out = new(), new()
            tp.delta_step(*qkvrb, b.lam, states[i], states[i], y.view(B, b.H, b.d), done=done)
            tp.norm_forward(self._norm(i + 1, B), x, y, z, x, n_out)
            n = n_out
        return self.head.forward(n, self.bias)


def train_to_follow(T=48, B=64, S=31, n=5, iterations=200, lr=0.01, seed=0):
    """Teach a policy to act on the mean of the last eight bars of the first features: actions drawn
    from it, advantages by how near they come, two clipped updates on each draw.  The mean squared
    distance of its means, per iteration."""
    g = torch.Generator("cuda").manual_seed(seed)
    policy = MatrixPolicy(S, n, H=2, d=32, blocks=2, dtype=torch.float32, seed=seed)
    opt = torch.optim.Adam(policy.parameters().values(), lr=lr)
    seen = []
    for _ in range(iterations):
        obs = torch.randn(T, B, -(-S // 32) * 32, generator=g, device="cuda")
        want = torch.stack([obs[max(0, t - 7):t + 1, :, :n].sum(0) for t in range(T)]) / 8 ** 0.5
        mu_ref = policy.forward(obs).clone()
        log_std_ref = policy.log_std.clone()
        z = torch.randn(T, B, n, generator=g, device="cuda")
        action = mu_ref + torch.exp(log_std_ref) * z
        logp = (-0.5 * z * z - log_std_ref).sum(2) - 0.5 * n * math.log(2 * math.pi)
        gain = -(action - want).square().sum(2)
        adv = (gain - gain.mean()) / gain.std()
        seen.append(float((mu_ref - want).square().mean()))
        for _ in range(2):
            mu = policy.forward(obs)
            _, dmu, dlog_std = policy.loss(mu, action, logp, adv, mu_ref, log_std_ref, kl_coef=0.01)
            grads = policy.gradients(dmu, dlog_std)
            for k, p in policy.parameters().items():
                p.grad = grads[k]
            opt.step()
            policy.refresh()
    return seen


if __name__ == "__main__":
    dist = train_to_follow()
    print(f"distance {dist[0]:.3f} -> {dist[-1]:.3f} in {len(dist)} iterations")
