"""One sequence policy fitted to an archive's elites.

Each elite of a policy archive (workload task MLP_SYNTH) is a small network that
acts for an episode and ends at its own descriptor.  This module rolls the
elites out, fits one policy to their episodes that is told the wanted descriptor
in its first token, and rolls that policy out token by token:

  python -m paper_2202_01258_amd.seq_policy            # needs the GPU

The policy is a stack of blocks; each adds to a residual stream what attention
over a window gives (the descriptor's token stays visible: one sink), then what
linear attention with a decay for each head gives.  It shows the operators of
`seq` as they are used together: under autograd for fitting, `*_forward` with a
filled cache for a prompt, `*_step` for single tokens, the 8-bit norm in front
of the projections of a rollout.
"""
from __future__ import annotations

import math

import torch

from . import seq

OBS, ACT, DESC = 27, 8, 4


# ---------------------------------------------------------------------------
# Episodes of the elites
# ---------------------------------------------------------------------------
def environment(archive):
    """A [obs, obs], B [obs, act] and s0 [obs] of an archive's synthetic dynamics."""
    env = archive.views()["env"]
    a, b = OBS * OBS, OBS * OBS + OBS * ACT
    return env[:a].view(OBS, OBS), env[a:b].view(OBS, ACT), env[b:b + OBS]


def elites(archive):
    """Genotypes [n, length] and descriptors [n, 4] of the filled cells."""
    archive.stream.synchronize()
    v = archive.views()
    cells = (v["key"] != 0).nonzero()[:, 0]
    return v["geno"][v["slot"][cells].long(), cells, :archive.n].clone(), v["desc"][cells].clone()


def episodes(geno, hid, env, steps):
    """States [n, steps, obs] before, and actions [n, steps, act] at, each step of each elite."""
    a_mat, b_mat, s0 = env
    n = geno.shape[0]
    shapes = [(hid, OBS), (hid,), (hid, hid), (hid,), (ACT, hid), (ACT,)]
    parts = torch.split(geno, [math.prod(s) for s in shapes], 1)
    w1, b1, w2, b2, w3, b3 = (p.reshape(n, *s) for p, s in zip(parts, shapes))
    s, states, actions = s0.expand(n, OBS), [], []
    for _ in range(steps):
        h = torch.tanh((w1 @ s[..., None])[..., 0] + b1)
        h = torch.tanh((w2 @ h[..., None])[..., 0] + b2)
        act = torch.tanh((w3 @ h[..., None])[..., 0] + b3)
        states.append(s)
        actions.append(act)
        s = torch.tanh(s @ a_mat.T + act @ b_mat.T)
    return torch.stack(states, 1), torch.stack(actions, 1)


def descriptors(states):
    """The descriptor of episodes [n, steps, obs] of states after each step."""
    return torch.sigmoid(states[..., 1:1 + DESC]).mean(1)


# ---------------------------------------------------------------------------
# The policy
# ---------------------------------------------------------------------------
class SequencePolicy(torch.nn.Module):
    """Token 0 holds the wanted descriptor, token t + 1 the state before step t;
    the output at token t + 1 is the action of step t.  Parameters are fp32, the
    tokens bfloat16."""

    def __init__(self, width=128, heads=2, blocks=2, window=64, device="cuda:0"):
        super().__init__()
        if width % heads or width // heads % 8:
            raise ValueError(f"width {width}: heads ({heads}) times a multiple of 8")
        self.width, self.heads, self.blocks, self.window, self.sinks = width, heads, blocks, window, 1
        self.dim = width // heads

        def weight(rows, cols, scale=1.0):
            w = torch.randn(rows, cols, device=device) * (scale / math.sqrt(rows))
            return torch.nn.Parameter(w)

        self.embed_desc, self.embed_obs = weight(DESC, width), weight(OBS, width)
        self.qkv = torch.nn.ParameterList(weight(width, 3 * width) for _ in range(2 * blocks))
        self.out = torch.nn.ParameterList(weight(width, width, 0.5) for _ in range(2 * blocks))
        self.norm = torch.nn.ParameterList(
            torch.nn.Parameter(torch.ones(width, device=device)) for _ in range(2 * blocks + 1))
        self.head = weight(width, ACT, 0.5)
        # memories of 8 to 512 steps
        horizon = 2.0 ** torch.linspace(3.0, 9.0, heads, device=device)
        self.register_buffer("log_decay", torch.log1p(-1.0 / horizon))

    def _split(self, x):
        """q, k and v, as slices of their projection."""
        x = x.view(*x.shape[:-1], 3 * self.heads, self.dim)
        return x[..., :self.heads, :], x[..., self.heads:2 * self.heads, :], x[..., 2 * self.heads:, :]

    def tokens(self, desc, states):
        """[n, 1 + steps, width] from descriptors [n, 4] and states [n, steps, obs]."""
        first = (desc - 0.5) @ self.embed_desc
        return torch.cat([first[:, None], states @ self.embed_obs], 1).to(torch.bfloat16)

    def forward(self, tokens, lengths=None):
        """Actions [n, tokens, act] (that of token 0 means nothing)."""
        low = torch.bfloat16
        stream, add = None, tokens
        for i in range(2 * self.blocks):
            y, stream = seq.residual_norm(add, stream, self.norm[i])
            q, k, v = self._split(y @ self.qkv[i].to(low))
            if i % 2 == 0:
                o = seq.window_attention(q, k, v, self.window, self.sinks, lengths)
            else:
                o, _ = seq.decay_attention(q, k, v, self.log_decay, lengths=lengths)
            add = o.flatten(-2) @ self.out[i].to(low)
        y, _ = seq.residual_norm(add, stream, self.norm[-1])
        return torch.tanh((y @ self.head.to(low)).float())


class Rollout:
    """A policy's state for `batch` episodes, one token at a time."""

    def __init__(self, policy: SequencePolicy, batch: int):
        self.policy, p = policy, policy
        dev, low = p.log_decay.device, torch.bfloat16
        self.pos = torch.zeros(batch, dtype=torch.int32, device=dev)
        self.cache = [seq.window_cache(batch, p.heads, p.dim, p.window, p.sinks, low, dev)
                      for _ in range(p.blocks)]
        self.state = [torch.zeros(batch, p.heads, p.dim, p.dim, device=dev) for _ in range(p.blocks)]
        self.qkv = [w.detach().to(low) for w in p.qkv]
        self.out = [w.detach().to(low) for w in p.out]
        self.norm = [w.detach().clone() for w in p.norm]
        self.head = p.head.detach().to(low)

    @torch.no_grad()
    def step(self, token, eight_bits=False):
        """Actions [batch, act] for one token [batch, width] of each episode.  With
        `eight_bits` the projections' inputs are e4m3 numbers with a scale per row
        (which the product of a row may be multiplied with afterwards).  The products
        themselves are bfloat16 here, so that shows the numbers and saves no time."""
        p, stream, add = self.policy, None, token
        for i in range(2 * p.blocks):
            if eight_bits:
                y, scale, stream = seq.residual_norm_fp8(add, stream, self.norm[i])
                proj = ((y.to(token.dtype) @ self.qkv[i]).float() * scale).to(token.dtype)
            else:
                y, stream, _ = seq.residual_norm_forward(add, stream, self.norm[i])
                proj = y @ self.qkv[i]
            q, k, v = p._split(proj)
            if i % 2 == 0:
                kc, vc = self.cache[i // 2]
                o = seq.window_attention_step(q, k, v, kc, vc, self.pos, p.window, p.sinks)
            else:
                o, _ = seq.decay_attention_step(q, k, v, p.log_decay, self.state[i // 2])
            add = o.flatten(-2) @ self.out[i]
        y, _, _ = seq.residual_norm_forward(add, stream, self.norm[-1])
        self.pos += 1
        return torch.tanh((y @ self.head).float())

    @torch.no_grad()
    def prompt(self, tokens, lengths=None):
        """Takes in the first tokens [batch, n, width] of each episode at once
        (`lengths`: how many of them each has, clamped to 0 .. n); the next `step`
        continues them."""
        p, stream, add = self.policy, None, tokens
        n = tokens.shape[1]
        for i in range(2 * p.blocks):
            y, stream, _ = seq.residual_norm_forward(add, stream, self.norm[i])
            q, k, v = p._split(y @ self.qkv[i])
            if i % 2 == 0:
                o, _ = seq.window_attention_forward(q, k, v, p.window, p.sinks, lengths)
                seq.window_cache_fill(k, v, *self.cache[i // 2], p.window, p.sinks, lengths)
            else:
                o, last = seq.decay_attention_forward(q, k, v, p.log_decay, lengths=lengths)
                self.state[i // 2].copy_(last)
            add = o.flatten(-2) @ self.out[i]
        self.pos.copy_(torch.full_like(self.pos, n) if lengths is None else lengths.clamp(0, n))


def fit(policy, desc, states, actions, iterations=200, batch=64, lr=2e-3, seed=0):
    """Fits the policy to the elites' episodes; returns the loss of each iteration."""
    gen = torch.Generator(device=desc.device)
    gen.manual_seed(seed)
    optimizer = torch.optim.Adam(policy.parameters(), lr=lr)
    losses = []
    for _ in range(iterations):
        pick = torch.randint(0, desc.shape[0], (batch,), generator=gen, device=desc.device)
        got = policy(policy.tokens(desc[pick], states[pick]))[:, 1:]
        loss = (got - actions[pick]).square().mean()
        optimizer.zero_grad(set_to_none=True)
        loss.backward()
        optimizer.step()
        losses.append(loss.detach())
    return torch.stack(losses)


@torch.no_grad()
def act(policy, desc, env, steps, eight_bits=False):
    """Closed loop: states [n, steps, obs] after each step of episodes with wanted descriptors."""
    a_mat, b_mat, s0 = env
    run = Rollout(policy, desc.shape[0])
    s, out = s0.expand(desc.shape[0], OBS), []
    run.step(((desc - 0.5) @ policy.embed_desc).to(torch.bfloat16), eight_bits)
    for _ in range(steps):
        a = run.step((s @ policy.embed_obs).to(torch.bfloat16), eight_bits)
        s = torch.tanh(s @ a_mat.T + a @ b_mat.T)
        out.append(s)
    return torch.stack(out, 1)


def main(generations=200, steps=100, iterations=400):
    from . import qd, workloads
    torch.manual_seed(0)
    # wide steps and small cells, so that elites of many descriptors are kept
    archive = qd.Archive(workloads.workload("mlp64_cvt_b8192", batch=2048, T=steps, C=10000,
                                            iso_sigma=0.1, line_sigma=0.1))
    archive.generations(1, generations)
    env = environment(archive)
    geno, desc = elites(archive)
    states, actions = episodes(geno, archive.w["hid"], env, steps)
    print(f"{desc.shape[0]} elites, {steps} steps", flush=True)
    policy = SequencePolicy()
    losses = fit(policy, desc, states, actions, iterations)
    print(f"mean squared error of actions: {float(losses[:10].mean()):.4f} -> {float(losses[-10:].mean()):.4f}", flush=True)
    spread = float((desc - desc.mean(0)).norm(dim=1).mean())
    for eight_bits in (False, True):
        got = descriptors(act(policy, desc, env, steps, eight_bits))
        off = float((got - desc).norm(dim=1).mean())
        print(f"closed loop{' (8 bits)' if eight_bits else ''}: mean distance to the wanted descriptor {off:.4f} "
              f"(elites lie {spread:.4f} around their mean)", flush=True)


if __name__ == "__main__":
    main()
