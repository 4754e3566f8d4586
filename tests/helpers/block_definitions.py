"""The selective block's operators in 64 bits, straight from their definitions (a row, a tap, an
element at a time), with the magnitudes that rounding errors are measured by.

Each function takes float64 tensors on the CPU and is differentiated by torch's autograd, so
gradients come from the definitions and from no formula of the library's.  `mags` runs
the same definition on absolute values: what it gives, and its gradients, are the sums of the
magnitudes of all terms.
"""
import torch


def silu(x):
    return x * torch.sigmoid(x)


def silu_slope_mag(x):
    """The magnitudes of the slope's two terms, s and x s (1 - s): they cancel at x = -1.278, where
    float32 leaves 2^-24 of each of them (1 + x (1 - s) is rounded relative to 1), so the slope's own
    size bounds nothing there."""
    s = torch.sigmoid(x)
    return s + x.abs() * s * torch.sigmoid(-x)


# ---------------------------------------------------------------------------
# Short causal convolution
# ---------------------------------------------------------------------------
def conv_rows(x, weight, bias, state, ends):
    """The sums p [b, t, w] (0 behind an episode's end) and the last states."""
    taps = weight.shape[0]
    p, last = [], []
    for i, n in enumerate(ends):
        rows = torch.cat([state[i], x[i, :n]])
        last.append(rows[n:])
        s = sum(weight[k] * rows[k:k + n] for k in range(taps)) + bias
        p.append(torch.cat([s, s.new_zeros(x.shape[1] - n, x.shape[2])]))
    return torch.stack(p), torch.stack(last)


def conv(x, weight, bias, state, ends, act, dy=None, dlast=None):
    """Outputs and gradients as {name: (value, magnitude)}."""
    leaves = {"dx": x, "dw": weight, "db": bias, "dstate": state}
    leaves = {k: v.detach().clone().requires_grad_() for k, v in leaves.items()}
    p, last = conv_rows(*leaves.values(), ends)
    live = torch.tensor([[t < n for t in range(x.shape[1])] for n in ends], dtype=x.dtype).view(*x.shape[:2], 1)
    y = (silu(p) if act else p) * live
    mleaves = {k: v.detach().abs().requires_grad_() for k, v in leaves.items()}
    mp, mlast = conv_rows(*mleaves.values(), ends)
    out = {"y": (y.detach(), (1.1 * mp.detach() if act else mp.detach()) * live), "last": (last.detach(), mlast.detach())}
    if dy is not None:
        loss = (y * dy).sum() + (last * dlast).sum()
        got = torch.autograd.grad(loss, list(leaves.values()))
        # silu's slope is below 1.1, its slope's below 0.5: the error of p moves g by half of it
        up = (1.1 + 0.5 * mp.detach()) if act else torch.ones_like(mp)
        mloss = (mp * (dy.abs() * up * live)).sum() + (mlast * dlast.abs()).sum()
        mag = torch.autograd.grad(mloss, list(mleaves.values()))
        out.update({k: (g, m) for k, g, m in zip(leaves, got, mag)})
    return out


# ---------------------------------------------------------------------------
# Selective state space scan
# ---------------------------------------------------------------------------
def scan_rows(u, dt, xt, a, b, c, skip, value, state, ends, rates):
    """o [b, t, w] and the last states.  `dt` is the step in the decays, `xt` that of the inputs;
    `a` multiplies dt where gradients are taken, `rates` is its value."""
    batch, length, width = u.shape
    o = []
    h = state
    on = torch.tensor([[float(t < n) for t in range(length)] for n in ends], dtype=u.dtype)
    for t in range(length):
        live = on[:, t, None, None]
        decay = torch.exp(dt[:, t, :, None] * rates)
        new = decay * h + (xt[:, t] * u[:, t])[..., None] * b[:, t, None]
        h = torch.where(live > 0, new, h)
        y = (h * c[:, t, None]).sum(-1) + skip * u[:, t]
        o.append(y * value[:, t] * on[:, t, None])
    return (torch.stack(o, 1) if o else u * 0), h


class _Decay(torch.autograd.Function):
    """exp(dt a) whose gradients take the magnitudes of dt and a."""

    @staticmethod
    def forward(ctx, dt, a):
        e = torch.exp(dt * a)
        ctx.save_for_backward(dt, a, e)
        return e

    @staticmethod
    def backward(ctx, g):
        dt, a, e = ctx.saved_tensors
        da = (g * e * dt.abs())
        return (g * e * a.abs()).sum(-1, keepdim=True), da.sum(0)


def scan(u, delta, a, b, c, skip, gate, bias, state, ends, do=None, dlast=None):
    """Outputs and gradients as {name: (value, magnitude)}; also the largest dt |a|."""
    batch, length, width = u.shape
    on = torch.tensor([[float(t < n) for t in range(length)] for n in ends], dtype=u.dtype).view(batch, length, 1)
    names = ["du", "ddelta", "da", "db", "dc", "dskip", "dgate", "dbias", "dstate"]
    leaves = [t.detach().clone().requires_grad_() for t in (u, delta, a, b, c, skip, gate, bias, state)]
    lu, ldelta, la, lb, lc, lskip, lgate, lbias, lstate = leaves
    raw = ldelta + lbias
    dt = torch.logaddexp(raw, torch.zeros_like(raw))
    o, last = scan_rows(lu, dt, dt, la, lb, lc, lskip, silu(lgate), lstate, ends, la)
    # magnitudes: every factor by itself
    m = [t.detach().abs().clone().requires_grad_() for t in (u, b, c, skip, state)]
    mu, mb, mc, mskip, mstate = m
    dt0 = dt.detach()
    mdt, mxt = dt0.clone().requires_grad_(), dt0.clone().requires_grad_()
    ma = a.detach().clone().requires_grad_()
    mvalue = silu(gate).abs().requires_grad_()
    h, mo = mstate, []
    for t in range(length):
        new = _Decay.apply(mdt[:, t, :, None], ma) * h + (mxt[:, t] * mu[:, t])[..., None] * mb[:, t, None]
        h = torch.where(on[:, t, None] > 0, new, h)
        mo.append(((h * mc[:, t, None]).sum(-1) + mskip * mu[:, t]) * mvalue[:, t] * on[:, t])
    mo = torch.stack(mo, 1) if mo else mu * 0
    out = {"o": (o.detach(), mo.detach()), "last": (last.detach(), h.detach())}
    if do is not None:
        got = torch.autograd.grad((o * do).sum() + (last * dlast).sum(), leaves, allow_unused=True)
        got = [torch.zeros_like(t) if g is None else g for g, t in zip(got, leaves)]
        to = [mu, mdt, mxt, ma, mb, mc, mskip, mvalue, mstate]
        mag = torch.autograd.grad((mo * do.abs()).sum() + (h * dlast.abs()).sum(), to, allow_unused=True)
        mag = [torch.zeros_like(t) if g is None else g for g, t in zip(mag, to)]
        slope = torch.sigmoid(raw.detach())
        mdelta = (mag[1] + mag[2]) * slope
        mags = [mag[0], mdelta, mag[3], mag[4], mag[5], mag[6], mag[7] * silu_slope_mag(gate), mdelta.sum((0, 1)), mag[8]]
        out.update({k: (g, v) for k, g, v in zip(names, got, mags)})
    return out, float((dt0[..., None] * a.abs()).max()) if dt0.numel() else 0.0


# ---------------------------------------------------------------------------
# Norms after and before a block
# ---------------------------------------------------------------------------
def branch(x, gate, residual, w1, w2, scale, eps, dy=None, dh=None):
    """Outputs and gradients as {name: (value, magnitude)}."""
    leaves = [t.detach().clone().requires_grad_() for t in (x, gate, residual, w1, w2)]
    lx, lg, lr, l1, l2 = leaves
    sx = torch.rsqrt((lx * lx).mean(-1, keepdim=True) + eps)
    n = lx * sx
    h = scale * lr + silu(lg) * n * l1
    sh = torch.rsqrt((h * h).mean(-1, keepdim=True) + eps)
    y = h * sh * l2
    # h's own terms may cancel: what they are rounded by reaches everything behind them
    mh = ((scale * lr).abs() + (silu(lg) * n * l1).abs()).detach()
    top = (mh * sh + (h * sh).abs() * (mh * h.abs()).mean(-1, keepdim=True) * sh * sh).detach()
    out = {"y": (y.detach(), top * l2.abs().detach()), "h": (h.detach(), mh), "rx": (sx.detach()[..., 0], sx.detach()[..., 0]),
           "rh": (sh.detach()[..., 0], (sh * (1 + (mh * h.abs()).mean(-1, keepdim=True) * sh * sh)).detach()[..., 0])}
    if dy is not None:
        got = torch.autograd.grad((y * dy).sum() + (h * dh).sum(), leaves)
        with torch.no_grad():
            e, m = (dy * l2).abs(), h.abs() * sh
            dot = (e * (m + top)).mean(-1, keepdim=True)
            # rh and m carry h's rounding, in relative terms by mh / rms
            loose = 1 + (mh * h.abs()).mean(-1, keepdim=True) * sh * sh
            mgh = dh.abs() + sh * loose * (e + (m + top) * dot)
            na, sg = n.abs(), silu(lg).abs()
            f = mgh * sg * l1.abs()
            mags = [sx * (f + na * (f * na).mean(-1, keepdim=True)), mgh * na * l1.abs() * (silu_slope_mag(lg) + 0.5),
                    abs(scale) * mgh, (mgh * sg * na).flatten(0, -2).sum(0), (dy.abs() * (m + top)).flatten(0, -2).sum(0)]
        out.update({k: (g, v) for k, g, v in zip(("dx", "dgate", "dresidual", "dw1", "dw2"), got, mags)})
    return out


# ---------------------------------------------------------------------------
# Philox4x32-10 and the draws
# ---------------------------------------------------------------------------
def philox(counter, key):
    """One block, in Python's integers."""
    c, k = list(counter), list(key)
    for _ in range(10):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [b >> 32 ^ c[1] ^ k[0], b & 0xFFFFFFFF, a >> 32 ^ c[3] ^ k[1], a & 0xFFFFFFFF]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def draws(elements, seed, step, site):
    """The 16-bit draws of the given elements (a list of places)."""
    seed, step = seed & (1 << 64) - 1, step & (1 << 64) - 1
    out = []
    for e in elements:
        w = philox((e // 8, site, step & 0xFFFFFFFF, step >> 32), (seed & 0xFFFFFFFF, seed >> 32))[e % 8 // 2]
        out.append(w >> 16 if e & 1 else w & 0xFFFF)
    return out
