"""One sequence policy fitted to an archive's elites.

Each elite of a policy archive (workload task MLP_SYNTH) is a small network that
acts for an episode and ends at its own descriptor.  This module rolls the
elites out, fits one policy to their episodes that is told the wanted descriptor
in its first token, and rolls that policy out token by token:

  python -m paper_2202_01258_amd.seq_policy            # needs the GPU

The policy is a stack of blocks; each adds to a residual stream what attention
over a window gives (the descriptor's token stays visible: one sink), then what
linear attention with a decay for each head gives.  A block may also hold a
selective scan behind a short convolution, which chooses by what it reads what it
remembers (`mixers`); branches may be normed and gated before they are added
(`post_norm`), and dropped out while fitting (`dropout`), as few elites are soon
learnt by heart:

  python -m paper_2202_01258_amd.seq_policy --mixers window,scan --post-norm --dropout 0.1

It shows the operators of `seq` as they are used together: under autograd for
fitting, `*_forward` with a filled cache for a prompt, `*_step` for single tokens,
the 8-bit norm in front of the projections of a rollout.
"""
from __future__ import annotations

import argparse
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
    tokens bfloat16.

    A block has a layer for each of `mixers`: "window", "decay" or "scan".  With
    `post_norm` a layer's output is normed and gated before it joins the stream, which is
    scaled by `residual_scale`; `dropout` is the share of each layer's output that is
    zero while the module is in training mode (its random state, `rng`, is advanced by fit)."""

    TAPS, STATES = 4, 16             # of the scan: taps of its convolution, states of a column

    def __init__(self, width=128, heads=2, blocks=2, window=64, device="cuda:0", mixers=("window", "decay"),
                 post_norm=False, residual_scale=1.0, dropout=0.0, seed=0):
        super().__init__()
        if width % heads or width // heads % 8:
            raise ValueError(f"width {width}: heads ({heads}) times a multiple of 8")
        if not mixers or any(m not in ("window", "decay", "scan") for m in mixers):
            raise ValueError(f"mixers {mixers}: of window, decay and scan")
        if not math.isfinite(residual_scale):
            raise ValueError(f"residual_scale {residual_scale}: a finite number")
        seq.dropout_threshold(dropout)       # refuses what the layers would
        self.width, self.heads, self.blocks, self.window, self.sinks = width, heads, blocks, window, 1
        self.dim = width // heads
        self.layers = list(mixers) * blocks
        self.post_norm, self.residual_scale, self.dropout = post_norm, residual_scale, dropout
        self.inner, self.rank = 2 * width, max(8, width // 16)

        def weight(rows, cols, scale=1.0):
            w = torch.randn(rows, cols, device=device) * (scale / math.sqrt(rows))
            return torch.nn.Parameter(w)

        # a layer's first product gives q, k and v, or a scan's input and gate; then the branch's gate
        into = [(2 * self.inner if m == "scan" else 3 * width) + (width if post_norm else 0) for m in self.layers]
        self.embed_desc, self.embed_obs = weight(DESC, width), weight(OBS, width)
        self.qkv = torch.nn.ParameterList(weight(width, n) for n in into)
        self.out = torch.nn.ParameterList(weight(self.inner if m == "scan" else width, width, 0.5) for m in self.layers)
        self.norm = torch.nn.ParameterList(
            torch.nn.Parameter(torch.ones(width, device=device)) for _ in range(len(self.layers) + 1))
        self.head = weight(width, ACT, 0.5)
        # memories of 8 to 512 steps
        horizon = 2.0 ** torch.linspace(3.0, 9.0, heads, device=device)
        self.register_buffer("log_decay", torch.log1p(-1.0 / horizon))
        if post_norm:
            self.branch = torch.nn.ParameterList(
                torch.nn.Parameter(torch.full((width,), 0.5, device=device)) for _ in self.layers)
        if "scan" in self.layers:
            self.scan = torch.nn.ModuleList(
                self._scan_weights(weight, device) if m == "scan" else torch.nn.Module() for m in self.layers)
        if dropout:
            self.register_buffer("rng", seq.dropout_rng(seed, 0, device))

    def _scan_weights(self, weight, device):
        """The convolution, the products that give the scan's steps, b and c, and its constants:
        rates of 1 to STATES, steps of 0.001 to 0.1."""
        m, inner, n = torch.nn.Module(), self.inner, self.STATES
        m.conv = weight(self.TAPS, inner)
        m.conv_bias = torch.nn.Parameter(torch.zeros(inner, device=device))
        m.small = weight(inner, self.rank + 2 * n)
        m.delta = weight(self.rank, inner, 0.1)
        step = torch.exp(torch.linspace(math.log(1e-3), math.log(0.1), inner, device=device))
        m.bias = torch.nn.Parameter(torch.log(torch.expm1(step)))
        m.log_rate = torch.nn.Parameter(torch.log(torch.arange(1.0, n + 1, device=device)).expand(inner, n).contiguous())
        m.skip = torch.nn.Parameter(torch.ones(inner, device=device))
        return m

    def _split(self, x):
        """q, k and v, as slices of their projection."""
        x = x[..., :3 * self.width].unflatten(-1, (3 * self.heads, self.dim))
        return x[..., :self.heads, :], x[..., self.heads:2 * self.heads, :], x[..., 2 * self.heads:, :]

    def _split_scan(self, x):
        """A scan's input and its gate."""
        return x[..., :self.inner], x[..., self.inner:2 * self.inner]

    def _split_small(self, x):
        """What the steps are made of, b and c."""
        return x.split([self.rank, self.STATES, self.STATES], -1)

    def tokens(self, desc, states):
        """[n, 1 + steps, width] from descriptors [n, 4] and states [n, steps, obs]."""
        first = (desc - 0.5) @ self.embed_desc
        return torch.cat([first[:, None], states @ self.embed_obs], 1).to(torch.bfloat16)

    def _mix(self, i, proj, lengths):
        """What layer i makes of its projection, in front of its last product."""
        low = proj.dtype
        if self.layers[i] == "scan":
            m = self.scan[i]
            u, gate = self._split_scan(proj)
            u, _ = seq.causal_conv(u, m.conv, m.conv_bias, lengths=lengths)
            steps, b, c = self._split_small(u @ m.small.to(low))
            o, _ = seq.selective_scan(u, steps @ m.delta.to(low), -m.log_rate.exp(), b, c, m.skip, gate, m.bias,
                                      lengths=lengths)
            return o
        q, k, v = self._split(proj)
        if self.layers[i] == "window":
            o = seq.window_attention(q, k, v, self.window, self.sinks, lengths)
        else:
            o, _ = seq.decay_attention(q, k, v, self.log_decay, lengths=lengths)
        return o.flatten(-2)

    def forward(self, tokens, lengths=None):
        """Actions [n, tokens, act] (that of token 0 means nothing)."""
        low = torch.bfloat16
        y, stream = seq.residual_norm(tokens, None, self.norm[0])
        for i in range(len(self.layers)):
            proj = y @ self.qkv[i].to(low)
            add = self._mix(i, proj, lengths) @ self.out[i].to(low)
            if self.dropout and self.training:
                add = seq.dropout(add, self.rng, self.dropout, site=i)
            if self.post_norm:
                y, stream = seq.branch_norm(add, proj[..., -self.width:], stream, self.branch[i], self.norm[i + 1],
                                            self.residual_scale)
            else:
                y, stream = seq.residual_norm(add, stream, self.norm[i + 1])
        return torch.tanh((y @ self.head.to(low)).float())


class Rollout:
    """A policy's state for `batch` episodes, one token at a time."""

    def __init__(self, policy: SequencePolicy, batch: int):
        self.policy, p = policy, policy
        dev, low = p.log_decay.device, torch.bfloat16
        self.pos = torch.zeros(batch, dtype=torch.int32, device=dev)
        count = p.layers.count
        # what each kind of layer remembers, in the order of the layers
        self.cache = [seq.window_cache(batch, p.heads, p.dim, p.window, p.sinks, low, dev) for _ in range(count("window"))]
        self.state = [torch.zeros(batch, p.heads, p.dim, p.dim, device=dev) for _ in range(count("decay"))]
        self.rows = [torch.zeros(batch, p.TAPS - 1, p.inner, dtype=low, device=dev) for _ in range(count("scan"))]
        self.scan = [torch.zeros(batch, p.inner, p.STATES, device=dev) for _ in range(count("scan"))]
        self.place = [p.layers[:i].count(m) for i, m in enumerate(p.layers)]
        self.qkv = [w.detach().to(low) for w in p.qkv]
        self.out = [w.detach().to(low) for w in p.out]
        self.norm = [w.detach().clone() for w in p.norm]
        self.head = p.head.detach().to(low)
        self.branch = [w.detach().clone() for w in p.branch] if p.post_norm else None
        self.weights = [self._scan_weights(m) for m, kind in zip(getattr(p, "scan", ()), p.layers) if kind == "scan"]

    @staticmethod
    def _scan_weights(m):
        copy = {k: getattr(m, k).detach().clone() for k in ("conv", "conv_bias", "bias", "skip")}
        low = {k: getattr(m, k).detach().to(torch.bfloat16) for k in ("small", "delta")}
        return dict(copy, **low, a=-m.log_rate.detach().exp())

    def _join(self, i, add, proj, stream):
        """The norm behind layer i and in front of the next."""
        p = self.policy
        if p.post_norm:
            y, stream, _ = seq.branch_norm_forward(add, proj[..., -p.width:], stream, self.branch[i], self.norm[i + 1],
                                                   p.residual_scale)
        else:
            y, stream, _ = seq.residual_norm_forward(add, stream, self.norm[i + 1])
        return y, stream

    @torch.no_grad()
    def step(self, token, eight_bits=False):
        """Actions [batch, act] for one token [batch, width] of each episode.  With
        `eight_bits` the projections' inputs are e4m3 numbers with a scale per row
        (which the product of a row may be multiplied with afterwards).  The products
        themselves are bfloat16 here, so that shows the numbers and saves no time."""
        p, stream, add, low = self.policy, None, token, token.dtype
        if eight_bits and p.post_norm:
            raise ValueError("eight_bits: not with post_norm, whose norm has no 8-bit output")
        if not eight_bits:
            y, stream, _ = seq.residual_norm_forward(token, None, self.norm[0])
        for i, kind in enumerate(p.layers):
            at = self.place[i]
            if eight_bits:
                y, scale, stream = seq.residual_norm_fp8(add, stream, self.norm[i])
                proj = ((y.to(low) @ self.qkv[i]).float() * scale).to(low)
            else:
                proj = y @ self.qkv[i]
            if kind == "scan":
                w = self.weights[at]
                u, gate = p._split_scan(proj)
                u, _ = seq.causal_conv_step(u, w["conv"], w["conv_bias"], self.rows[at])
                steps, b, c = p._split_small(u @ w["small"])
                o, _ = seq.selective_scan_step(u, steps @ w["delta"], w["a"], b, c, self.scan[at], w["skip"], gate, w["bias"])
            else:
                q, k, v = p._split(proj)
                if kind == "window":
                    kc, vc = self.cache[at]
                    o = seq.window_attention_step(q, k, v, kc, vc, self.pos, p.window, p.sinks)
                else:
                    o, _ = seq.decay_attention_step(q, k, v, p.log_decay, self.state[at])
                o = o.flatten(-2)
            add = o @ self.out[i]
            if not eight_bits:
                y, stream = self._join(i, add, proj, stream)
        if eight_bits:
            y, _, _ = seq.residual_norm_forward(add, stream, self.norm[-1])
        self.pos += 1
        return torch.tanh((y @ self.head).float())

    @torch.no_grad()
    def prompt(self, tokens, lengths=None):
        """Takes in the first tokens [batch, n, width] of each episode at once
        (`lengths`: how many of them each has, clamped to 0 .. n); the next `step`
        continues them."""
        p, n = self.policy, tokens.shape[1]
        y, stream, _ = seq.residual_norm_forward(tokens, None, self.norm[0])
        for i, kind in enumerate(p.layers):
            at = self.place[i]
            proj = y @ self.qkv[i]
            if kind == "scan":
                w = self.weights[at]
                u, gate = p._split_scan(proj)
                u, rows = seq.causal_conv_forward(u, w["conv"], w["conv_bias"], lengths=lengths)
                steps, b, c = p._split_small(u @ w["small"])
                o, last, _ = seq.selective_scan_forward(u, steps @ w["delta"], w["a"], b, c, w["skip"], gate, w["bias"],
                                                        lengths=lengths)
                self.rows[at].copy_(rows)
                self.scan[at].copy_(last)
            else:
                q, k, v = p._split(proj)
                if kind == "window":
                    o, _ = seq.window_attention_forward(q, k, v, p.window, p.sinks, lengths)
                    seq.window_cache_fill(k, v, *self.cache[at], p.window, p.sinks, lengths)
                else:
                    o, last = seq.decay_attention_forward(q, k, v, p.log_decay, lengths=lengths)
                    self.state[at].copy_(last)
                o = o.flatten(-2)
            y, stream = self._join(i, o @ self.out[i], proj, stream)
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
        if policy.dropout:
            policy.rng[1] += 1
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


def main(generations=200, steps=100, iterations=400, **how):
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
    policy = SequencePolicy(**how)
    losses = fit(policy, desc, states, actions, iterations)
    print(f"mean squared error of actions: {float(losses[:10].mean()):.4f} -> {float(losses[-10:].mean()):.4f}", flush=True)
    spread = float((desc - desc.mean(0)).norm(dim=1).mean())
    for eight_bits in (False, True)[:1 if policy.post_norm else 2]:
        got = descriptors(act(policy, desc, env, steps, eight_bits))
        off = float((got - desc).norm(dim=1).mean())
        print(f"closed loop{' (8 bits)' if eight_bits else ''}: mean distance to the wanted descriptor {off:.4f} "
              f"(elites lie {spread:.4f} around their mean)", flush=True)


if __name__ == "__main__":
    args = argparse.ArgumentParser(description="fits one policy to an archive's elites and rolls it out")
    args.add_argument("--mixers", default="window,decay", help="a block's layers, of window, decay and scan")
    args.add_argument("--post-norm", action="store_true")
    args.add_argument("--dropout", type=float, default=0.0)
    args = args.parse_args()
    main(mixers=tuple(args.mixers.split(",")), post_norm=args.post_norm, dropout=args.dropout)
