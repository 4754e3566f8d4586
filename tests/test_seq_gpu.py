"""The sequence policy's operators on the GPU against their definitions in 64 bits.

Tolerances are bounds worked out from the kernels' roundings, element by
element, with u the unit roundoff of the tensors' type (2^-8 bfloat16, 2^-11
float16, 2^-24 float32).  What is rounded to that type is: the result; the
softmax weights and the score gradients in front of a matrix product; the
products of rows and the state in front of the decay's output products.  All
else is fp32, whose share is taken as SINGLE times the sum of the terms'
magnitudes: some hundred additions and a few operations on each term.
"""
import math

import pytest

torch = pytest.importorskip("torch")

from paper_2202_01258_amd import seq as S  # noqa: E402

pytestmark = pytest.mark.gpu

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
U = {BF16: 2.0 ** -8, F16: 2.0 ** -11, F32: 2.0 ** -24}
TINY = {BF16: 0.0, F16: 2.0 ** -25, F32: 0.0}      # half of the least float16 above 0: rounding of what is below its normal range
SINGLE = 2.0 ** -16
FLUSH = 2.0 ** -126        # weights below the least normal number are 0


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def rand(*shape, dtype=F32, seed=0, scale=1.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 1000003 + sum(shape))
    return (torch.randn(*shape, generator=g, device="cuda") * scale).to(dtype)


def within(got, want, bound, what):
    assert got.shape == want.shape, (what, got.shape, want.shape)
    err = (got.double() - want).abs()
    bad = ~(err <= bound)
    assert not bad.any(), (f"{what}: {int(bad.sum())} of {bad.numel()} outside, worst by "
                           f"{float((err / bound.clamp(min=1e-300))[bad].max()):.3g} times, first at "
                           f"{bad.nonzero()[0].tolist()}")


# ---------------------------------------------------------------------------
# Norm
# ---------------------------------------------------------------------------
EPS = 1e-6
NORM_SHAPES = [(1, 1), (5, 7), (3, 64), (9, 128), (1, 512), (17, 520), (6, 777), (4, 1000), (3, 1024), (5, 2048),
               (3, 2056), (2, 4096), (3, 5000), (2, 8192), (2, 9001), (2, 20000)]


def norm_inputs(rows, width, dtype, wdtype, seed=1):
    return (rand(rows, width, dtype=dtype, seed=seed), rand(rows, width, dtype=dtype, seed=seed + 1, scale=2.0),
            (1 + 0.2 * rand(width, seed=seed + 2)).to(wdtype))


def norm_exact(x, r, w, eps=EPS):
    h = x.double() + (r.double() if r is not None else 0)
    rstd = 1 / torch.sqrt((h * h).mean(-1, keepdim=True) + eps)
    return h, rstd, h * rstd * w.double()


@pytest.mark.parametrize("rows,width", NORM_SHAPES)
@pytest.mark.parametrize("dtype,wdtype", [(BF16, BF16), (F16, F32), (F32, F32)])
def test_norm_forward(rows, width, dtype, wdtype):
    x, r, w = norm_inputs(rows, width, dtype, wdtype)
    y, h, rstd = S.residual_norm_forward(x, r, w, eps=EPS)
    eh, es, ey = norm_exact(x, r, w)
    within(h, eh, U[dtype] * eh.abs() + TINY[dtype], "h")
    within(rstd, es[:, 0], SINGLE * es[:, 0], "rstd")
    within(y, ey, (U[dtype] + SINGLE) * ey.abs() + TINY[dtype], "y")
    y2, h2, _ = S.residual_norm_forward(x, None, w, eps=EPS)
    assert torch.equal(h2, x)
    e2 = norm_exact(x, None, w)[2]
    within(y2, e2, (U[dtype] + SINGLE) * e2.abs() + TINY[dtype], "y without a residual")


def strided(t, how):
    """The same values in another layout."""
    rows, width = t.shape
    if how == "wide":                                  # a column range of a wider tensor
        big = torch.full((rows, width + 24), float("nan"), dtype=t.dtype, device=t.device)
        big[:, 8:8 + width] = t
        return big[:, 8:8 + width]
    if how == "odd":                                   # no row at a multiple of 16 bytes
        big = torch.full((rows, width + 3), float("nan"), dtype=t.dtype, device=t.device)
        big[:, 1:1 + width] = t
        return big[:, 1:1 + width]
    return t.t().contiguous().t()                      # columns apart: copied by the binding


@pytest.mark.parametrize("how", ["wide", "odd", "columns"])
@pytest.mark.parametrize("width", [128, 1024, 9216])
def test_norm_layouts(how, width):
    x, r, w = norm_inputs(6, width, BF16, BF16)
    want = S.residual_norm_forward(x, r, w)
    got = S.residual_norm_forward(strided(x, how), strided(r, how), w)
    _, _, ey = norm_exact(x, r, w)
    assert torch.equal(got[1], want[1])
    within(got[0], ey, (U[BF16] + SINGLE) * ey.abs(), "y")
    for group in (0, 128):
        q, s, h = S.residual_norm_fp8(strided(x, how), strided(r, how), w, group=group)
        check_fp8(q, s, h, x, r, w, group)
    dy, dh = rand(6, width, dtype=BF16, seed=7), rand(6, width, dtype=BF16, seed=8)
    check_norm_backward(strided(dy, how), strided(dh, how), want[1], want[2], w, dy, dh)


def check_fp8(q, s, h, x, r, w, group):
    eh, _, ey = norm_exact(x, r, w)
    rows, width = x.shape
    within(h, eh, U[h.dtype] * eh.abs() + TINY[h.dtype], "h")
    g = ey.view(rows, -1, group or width)
    top = g.abs().amax(-1)
    es = torch.where(top == 0, 1.0, top.clamp(min=2.0 ** -100) / 448)
    within(s, es, SINGLE * es, "scale")
    assert q.dtype == torch.float8_e4m3fn
    # 4 significant bits, or steps of 2^-9 below 2^-6; the quotient itself is fp32
    e = g / es[..., None]
    got = q.double().view_as(g)
    within(got, e, (2.0 ** -4 + SINGLE) * e.abs() + 2.0 ** -10, "q")
    assert got.abs().max() <= 448


@pytest.mark.parametrize("rows,width", NORM_SHAPES)
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
def test_norm_fp8_rows(rows, width, dtype):
    x, r, w = norm_inputs(rows, width, dtype, dtype, seed=3)
    q, s, h = S.residual_norm_fp8(x, r, w, eps=EPS)
    assert s.shape == (rows, 1)
    check_fp8(q, s, h, x, r, w, 0)


@pytest.mark.parametrize("rows,width", [(1, 128), (5, 256), (3, 640), (3, 1024), (2, 2048), (2, 4096), (2, 8192), (2, 12800)])
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
def test_norm_fp8_groups(rows, width, dtype):
    x, r, w = norm_inputs(rows, width, dtype, dtype, seed=3)
    q, s, h = S.residual_norm_fp8(x, r, w, eps=EPS, group=128)
    assert s.shape == (rows, width // 128)
    check_fp8(q, s, h, x, r, w, 128)


@pytest.mark.parametrize("width", [128, 1024, 8192, 16384])
def test_norm_special_values(width):
    """Zero rows, rows whose squares vanish in fp32, not-a-number and infinity."""
    x = rand(6, width, dtype=F32, seed=5)
    x[0] = 0
    x[1] = 1e-30
    x[2, 3] = float("nan")
    x[3, 5] = float("inf")
    w = torch.ones(width, device="cuda")
    y, h, _ = S.residual_norm_forward(x, None, w, eps=EPS)
    assert (y[0] == 0).all() and torch.allclose(y[1], x[1] * 1e3, rtol=1e-5)
    assert y[2].isnan().all() and (y[3].isnan().sum() == 1) and (y[3, :5] == 0).all()
    assert y[4:].isfinite().all()
    for group in (0, 128):
        q, s, _ = S.residual_norm_fp8(x, None, w, eps=EPS, group=group)
        q = q.float()
        assert (q[0] == 0).all() and (s[0] == 1).all()
        assert (q[1] == 448).all()
        assert q[2].isnan().all()
        assert q[3, 5].isnan() and (q[3, :5] == 0).all()
        assert q[4:].isfinite().all()


def check_norm_backward(dy, dh, h, rstd, w, dy0=None, dh0=None):
    dtype = h.dtype
    dx, dw = S.residual_norm_backward(dy, dh, h, rstd, w)
    gy = (dy if dy0 is None else dy0).double()
    gh = 0 if dh is None else (dh if dh0 is None else dh0).double()
    h, s, wd = h.double(), rstd.double()[:, None], w.double()
    g = gy * wd
    dot = (g * h).mean(-1, keepdim=True)
    want = gh + s * (g - h * s * s * dot)
    size = (gh.abs() if dh is not None else 0) + s * (g.abs() + h.abs() * s * s * (g * h).abs().mean(-1, keepdim=True))
    within(dx, want, U[dtype] * want.abs() + SINGLE * size + TINY[dtype], "dx")
    t = gy * h * s
    within(dw, t.sum(0), U[w.dtype] * t.sum(0).abs() + SINGLE * t.abs().sum(0) + TINY[w.dtype], "dweight")


@pytest.mark.parametrize("rows,width", NORM_SHAPES + [(2100, 24), (1500, 333), (700, 4096)])
@pytest.mark.parametrize("dtype,wdtype", [(BF16, BF16), (F16, F32), (F32, F32)])
def test_norm_backward(rows, width, dtype, wdtype):
    x, r, w = norm_inputs(rows, width, dtype, wdtype)
    _, h, rstd = S.residual_norm_forward(x, r, w)
    dy, dh = rand(rows, width, dtype=dtype, seed=7), rand(rows, width, dtype=dtype, seed=8)
    check_norm_backward(dy, dh, h, rstd, w)
    check_norm_backward(dy, None, h, rstd, w)


def test_norm_without_rows():
    x = torch.empty(0, 64, device="cuda")
    w = torch.ones(64, device="cuda")
    y, h, rstd = S.residual_norm_forward(x, x, w)
    assert y.shape == h.shape == (0, 64) and rstd.shape == (0,)
    dx, dw = S.residual_norm_backward(x, x, h, rstd, w)
    assert dx.shape == (0, 64) and (dw == 0).all()


def test_norm_gradient_against_differences():
    """fp32: the derivative along a direction from two calls.  The step's
    second-order share is step^2 / 6 of a third derivative of order 1; fp32
    rounding of some thousand values gives 2^-24 * sqrt(3000) / step."""
    x, r, w = norm_inputs(30, 100, F32, F32)
    gy, gh, d = rand(30, 100, seed=9), rand(30, 100, seed=10), rand(30, 100, seed=11)
    xs = [t.clone().requires_grad_() for t in (x, r, w)]
    y, h = S.residual_norm(*xs)
    (y * gy).sum().add((h * gh).sum()).backward()
    assert torch.equal(xs[0].grad, xs[1].grad)
    step = 2.0 ** -7

    def loss(x, w):
        y, h, _ = S.residual_norm_forward(x, r, w)
        return float((y.double() * gy).sum() + (h.double() * gh).sum())

    got = float((xs[0].grad.double() * d).sum())
    want = (loss(x + step * d, w) - loss(x - step * d, w)) / (2 * step)
    assert abs(got - want) <= 2e-3 * float((xs[0].grad.double() * d).norm())
    dw = rand(100, seed=12)
    got = float((xs[2].grad.double() * dw).sum())
    want = (loss(x, w + step * dw) - loss(x, w - step * dw)) / (2 * step)
    assert abs(got - want) <= 2e-3 * float((xs[2].grad.double() * dw).norm())


# ---------------------------------------------------------------------------
# Window attention
# ---------------------------------------------------------------------------
def qkv(b, t, hq, hkv, d, dtype, layout="fused", seed=1):
    if layout == "fused":                              # slices of one projection
        p = rand(b, t, hq + 2 * hkv, d, dtype=dtype, seed=seed)
        return p[:, :, :hq], p[:, :, hq:hq + hkv], p[:, :, hq + hkv:]
    if layout == "heads":                              # heads outside of rows
        return tuple(rand(b, n, t, d, dtype=dtype, seed=seed + i).transpose(1, 2) for i, n in enumerate((hq, hkv, hkv)))
    if layout == "time":                               # rows outside of the batch
        return tuple(rand(t, b, n, d, dtype=dtype, seed=seed + i).transpose(0, 1) for i, n in enumerate((hq, hkv, hkv)))
    if layout == "odd":                                # rows that are not aligned: copied by the binding
        return tuple(rand(b, t, n, d + 3, dtype=dtype, seed=seed + i)[..., 1:1 + d] for i, n in enumerate((hq, hkv, hkv)))
    return tuple(rand(b, t, n, d, dtype=dtype, seed=seed + i) for i, n in enumerate((hq, hkv, hkv)))


def window_exact(q, k, v, window, sinks, lengths=None, g=None, scale=None):
    """Results and bounds in 64 bits: {"o": (value, bound), ...}."""
    dtype = q.dtype
    u, tiny = U[dtype], TINY[dtype]
    b, t, hq, d = q.shape
    hkv = k.shape[2]
    c = d ** -0.5 if scale is None else scale
    n = torch.full((b,), t, device="cuda") if lengths is None else lengths.long().clamp(0, t)
    i = torch.arange(t, device="cuda")
    live = (i < n[:, None])[:, None, :, None]

    def rows(x, h):
        x = x.double().transpose(1, 2)
        x = torch.where(live, x, 0.0)
        return x.repeat_interleave(hq // h, 1).contiguous()

    Q, K, V = rows(q, hq), rows(k, hkv), rows(v, hkv)
    gap = i[:, None] - i
    seen = (gap >= 0) & ((gap < window) | (i < sinks)) & live
    s = (Q @ K.transpose(2, 3).contiguous() * c).masked_fill(~seen, -math.inf)
    lse = s.logsumexp(-1)
    p = torch.exp(s - lse.clamp(min=-1e300)[..., None])
    o = p @ V
    # weights are rounded relative to a sum of at least 1
    eo = u * o.abs() + (u + SINGLE) * (p @ V.abs()) + (tiny + FLUSH) * (1 + seen.double() @ V.abs())

    def home(x, h):
        x = x.view(b, h, hq // h, t, -1).sum(2)
        return x.transpose(1, 2)

    out = {"o": (home(o, hq), home(eo, hq)), "lse": (lse, SINGLE * (1 + s.abs().masked_fill(~seen, 0).amax(-1)))}
    if g is not None:
        G = rows(g, hq)
        VT = V.transpose(2, 3).contiguous()
        dp = G @ VT
        delta = (G * o).sum(-1, keepdim=True)
        ds = p * (dp - delta)
        # what the score's gradient is off by: its own rounding, o's in delta, fp32
        eds = (u * ds.abs() + p * (G.abs() * eo).sum(-1, keepdim=True) + tiny * seen
               + FLUSH * seen * (1 + dp.abs() + delta.abs())
               + SINGLE * p * (G.abs() @ VT.abs() + (G.abs() * o.abs()).sum(-1, keepdim=True)))
        PT, dsT, edsT = (x.transpose(2, 3).contiguous() for x in (p, ds, eds))
        dq, dk, dv = c * (ds @ K), c * (dsT @ Q), PT @ G
        edq = c * (eds @ K.abs())
        edk = c * (edsT @ Q.abs())
        edv = (u + SINGLE) * (PT @ G.abs()) + (tiny + FLUSH) * (seen.double().transpose(2, 3).contiguous() @ G.abs())
        for name, x, e, h in (("dq", dq, edq, hq), ("dk", dk, edk, hkv), ("dv", dv, edv, hkv)):
            x = home(x, h)
            out[name] = (x, u * x.abs() + home(e, h) + tiny + FLUSH)
    return out


def check_window(q, k, v, window, sinks, lengths=None, scale=None, backward=True):
    g = rand(*q.shape, dtype=q.dtype, seed=77) if backward else None
    o, lse = S.window_attention_forward(q, k, v, window, sinks, lengths, scale)
    want = window_exact(q, k, v, window, sinks, lengths, g, scale)
    within(o, *want["o"], "o")
    dead = want["lse"][0] == -math.inf
    assert torch.equal(lse == -math.inf, dead)
    within(lse[~dead], want["lse"][0][~dead], want["lse"][1][~dead], "lse")
    if backward:
        grads = S.window_attention_backward(g, q, k, v, o, lse, window, sinks, lengths, scale)
        for name, got in zip(("dq", "dk", "dv"), grads):
            within(got, *want[name], name)
        again = S.window_attention_backward(g, q, k, v, o, lse, window, sinks, lengths, scale)
        for a, b in zip(grads, again):
            assert torch.equal(a, b)


@pytest.mark.parametrize("t", [1, 2, 31, 63, 64, 65, 127, 128, 129, 300])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 2), (33, 0), (64, 1), (100, 70), (1000, 3), (50, 1000)])
def test_window_lengths_and_masks(t, window, sinks):
    check_window(*qkv(2, t, 2, 1, 64, BF16), window, sinks)


@pytest.mark.parametrize("d", [8, 32, 40, 64, 72, 80, 128])
@pytest.mark.parametrize("hq,hkv", [(1, 1), (3, 1), (4, 2), (8, 8)])
@pytest.mark.parametrize("dtype", [BF16, F16])
def test_window_heads_and_dims(d, hq, hkv, dtype):
    check_window(*qkv(2, 150, hq, hkv, d, dtype), 40, 5)


@pytest.mark.parametrize("d", [16, 24, 56, 88, 96, 104, 120])
@pytest.mark.parametrize("dtype", [BF16, F16])
def test_window_widths_around_a_step(d, dtype):
    """Products are formed of 32, 64, 96 or 128 columns, whichever hold the head."""
    check_window(*qkv(2, 140, 4, 2, d, dtype), 45, 3)
    check_window(*qkv(1, 700, 2, 1, d, dtype, "odd"), 700, 0, torch.tensor([650], dtype=torch.int32, device="cuda"))


@pytest.mark.parametrize("hq,hkv", [(4, 1), (6, 1), (6, 2), (12, 3), (8, 1), (16, 2)])
@pytest.mark.parametrize("d", [64, 128])
def test_window_head_groups(hq, hkv, d):
    """Groups of 2, 3, 4, 6 and 8 heads: one, two or four of them share a workgroup."""
    q, k, v = qkv(3, 170, hq, hkv, d, BF16)
    check_window(q, k, v, 37, 2)
    check_window(q, k, v, 1000, 0, torch.tensor([170, 33, 96], dtype=torch.int32, device="cuda"))


@pytest.mark.parametrize("layout", ["plain", "heads", "time", "odd"])
@pytest.mark.parametrize("d", [64, 128])
def test_window_layouts(layout, d):
    check_window(*qkv(3, 133, 4, 2, d, BF16, layout), 50, 3)


def test_window_broadcast_keys():
    """One key head spread by a stride of 0 over the batch."""
    q, k, v = qkv(3, 100, 2, 2, 64, BF16, "plain")
    k, v = (x[:1].expand(3, -1, -1, -1) for x in (k, v))
    check_window(q, k, v, 30, 2)


@pytest.mark.parametrize("d", [64, 128])
def test_window_ragged(d):
    q, k, v = (x.contiguous() for x in qkv(7, 200, 4, 2, d, F16))
    lengths = torch.tensor([200, 0, 1, 64, 65, 199, 130], dtype=torch.int32, device="cuda")
    # what is behind a length is never looked at
    for i, n in enumerate(lengths.tolist()):
        for x in (q, k, v):
            x[i, n:] = float("nan")
    check_window(q, k, v, 70, 3, lengths)
    # lengths outside of the tensor count as none and as all
    wild = torch.tensor([500, -3, 1, 64, 65, 199, 130], dtype=torch.int32, device="cuda")
    a = S.window_attention_forward(q, k, v, 70, 3, lengths)
    b = S.window_attention_forward(q, k, v, 70, 3, wild)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("t,window,sinks,b,hq,hkv,d", [
    (1500, 100, 0, 1, 1, 1, 64), (1500, 100, 130, 1, 2, 1, 64), (2500, 2000, 5, 1, 1, 1, 128),
    (1030, 300, 1, 1, 6, 1, 128)])
def test_window_few_heads(t, window, sinks, b, hq, hkv, d):
    """Key blocks whose work is cut into pieces."""
    check_window(*qkv(b, t, hq, hkv, d, BF16), window, sinks)


@pytest.mark.parametrize("b,hkv", [(1, 1), (3, 1), (2, 4), (9, 1), (4, 4), (17, 1), (5, 5)])
@pytest.mark.parametrize("window", [20, 300])
def test_window_order_of_work(b, hkv, window):
    """One, few and many lists, numbers of them that divide by eight and that do not:
    workgroups take their work in another order where lengths are given, results stay."""
    q, k, v = qkv(b, 300, 2 * hkv, hkv, 64, BF16)
    check_window(q, k, v, window, 2)
    whole = torch.full((b,), 300, dtype=torch.int32, device="cuda")
    o, lse = S.window_attention_forward(q, k, v, window, 2)
    for x, y in zip((o, lse), S.window_attention_forward(q, k, v, window, 2, whole)):
        assert torch.equal(x, y)
    do = rand(*o.shape, dtype=BF16, seed=9)
    for x, y in zip(S.window_attention_backward(do, q, k, v, o, lse, window, 2),
                    S.window_attention_backward(do, q, k, v, o, lse, window, 2, whole)):
        assert torch.equal(x, y)
    lengths = torch.tensor([(i * 131 + 77) % 301 for i in range(b)], dtype=torch.int32, device="cuda")
    check_window(q, k, v, window, 2, lengths)


def test_window_many_heads():
    """Key blocks that are not cut."""
    check_window(*qkv(40, 140, 8, 8, 64, BF16), 60, 2)


@pytest.mark.parametrize("scale", [0.01, 1.0])
def test_window_scale_and_large_scores(scale):
    """Scores up to some hundred: the maximum moves from tile to tile."""
    q, k, v = qkv(1, 400, 2, 2, 64, BF16, "plain")
    ramp = torch.linspace(0.1, 4.0, 400, device="cuda").to(BF16)[:, None, None]
    check_window(q * 2, k * ramp, v, 333, 3, scale=scale)


def test_window_gradient_against_differences():
    """Along a direction, from two calls of the forward pass in float16.  Inputs
    and steps are multiples of 2^-6, so that all of them are exact; o's rounding
    (2^-11 of values around 0.5, random) over the step gives a deviation of
    2^-11 * 0.5 * |g| / (sqrt(6) step), of which 6 are allowed, and the step's third-order
    share is some percent."""
    b, t, h, d = 2, 90, 2, 64
    q, k, v = ((torch.randint(-64, 65, (b, t, h, d), device="cuda", generator=torch.Generator("cuda").manual_seed(i)) / 64).to(F16)
               for i in range(3))
    g = rand(b, t, h, d, dtype=F16, seed=5)
    xs = [x.clone().requires_grad_() for x in (q, k, v)]
    S.window_attention(*xs, window=40, sinks=2, scale=0.25).backward(g)
    step = 2.0 ** -4
    for i in range(3):
        d_ = (torch.randint(-1, 2, (b, t, h, d), device="cuda", generator=torch.Generator("cuda").manual_seed(9 + i)) * step).to(F16)

        def loss(sign):
            y = [q, k, v]
            y[i] = y[i] + sign * d_
            return float((S.window_attention_forward(*y, 40, 2, scale=0.25)[0].double() * g).sum())

        got = float((xs[i].grad.double() * d_).sum())
        want = (loss(1) - loss(-1)) / 2
        noise = 2.0 ** -11 * 0.5 * float(g.double().norm()) / math.sqrt(6)
        size = float((xs[i].grad.double() * d_).norm())
        assert abs(got - want) <= 6 * noise + 0.1 * size, (i, got, want, noise, size)


def step_exact(q, k_rows, v_rows, window, sinks, pos):
    """o of each batch element from all of its rows so far ([b][pos + 1, hkv, d])."""
    b, hq, d = q.shape
    out = torch.zeros(b, hq, d, dtype=torch.float64, device="cuda")
    bound = torch.zeros_like(out)
    u, tiny = U[q.dtype], TINY[q.dtype]
    for i in range(b):
        p = pos[i]
        if p < 0:
            continue
        j = torch.arange(p + 1, device="cuda")
        seen = (p - j < window) | (j < sinks)
        group = hq // k_rows[i].shape[1]
        K = k_rows[i][:p + 1][seen].double().transpose(0, 1).repeat_interleave(group, 0)
        V = v_rows[i][:p + 1][seen].double().transpose(0, 1).repeat_interleave(group, 0)
        w = torch.softmax((K * q[i].double()[:, None]).sum(-1) * d ** -0.5, -1)[..., None]
        out[i] = (w * V).sum(1)
        bound[i] = u * out[i].abs() + (u + SINGLE) * (w * V.abs()).sum(1) + tiny * (1 + V.abs().sum(1))
    return out, bound


@pytest.mark.parametrize("window,sinks,d,hq,hkv,dtype", [
    (1, 0, 64, 2, 2, BF16), (5, 2, 64, 4, 2, BF16), (31, 0, 32, 2, 1, F16), (32, 1, 128, 8, 1, F16),
    (150, 3, 80, 20, 1, BF16), (97, 64, 128, 40, 2, BF16), (1700, 16, 128, 4, 2, BF16), (3000, 0, 64, 1, 1, F16)])
def test_window_steps_after_a_prompt(window, sinks, d, hq, hkv, dtype):
    """Prompts of all ages into the cache, then tokens; the cache's unused slots hold not-a-number."""
    ages = sorted({0, 1, 2, sinks, sinks + 1, window, window + sinks - 1, window + sinks, window + sinks + 1,
                   2 * window + sinks + 3})
    b, t = len(ages) + 1, ages[-1] + 4
    k_all, v_all = rand(b, t, hkv, d, dtype=dtype, seed=3), rand(b, t, hkv, d, dtype=dtype, seed=4)
    kc, vc = S.window_cache(b, hkv, d, window, sinks, dtype)
    kc.fill_(float("nan"))
    vc.fill_(float("nan"))
    lengths = torch.tensor(ages + [7], dtype=torch.int32, device="cuda")
    S.window_cache_fill(k_all, v_all, kc, vc, window, sinks, lengths)
    for step in range(3):
        pos = [a + step for a in ages] + [-1]
        at = torch.tensor(pos, device="cuda")
        rows = torch.arange(b, device="cuda")
        q = rand(b, hq, d, dtype=dtype, seed=50 + step)
        kept = kc[-1].clone()
        o = S.window_attention_step(q, k_all[rows, at], v_all[rows, at], kc, vc, at.to(torch.int32), window, sinks)
        within(o, *step_exact(q, k_all, v_all, window, sinks, pos), f"o at step {step}")
        assert (o[-1] == 0).all() and torch.equal(kc[-1].isnan(), kept.isnan())
        for i, p in enumerate(pos[:-1]):
            slot = p if p < sinks else sinks + (p - sinks) % window
            assert torch.equal(kc[i, :, slot], k_all[i, p]) and torch.equal(vc[i, :, slot], v_all[i, p])


@pytest.mark.parametrize("window,sinks,d,hq,hkv,dtype", [
    (20000, 3, 128, 20, 1, BF16), (33000, 0, 64, 2, 1, F16), (6000, 70, 72, 4, 2, BF16), (1200, 81, 64, 3, 3, F16), (1199, 81, 64, 3, 3, F16)])
def test_window_step_ranges(window, sinks, d, hq, hkv, dtype):
    """Few heads over long caches, whose slots are cut into many ranges, most of them
    empty for some positions; and the sizes on both sides of the first cut."""
    slots = window + sinks
    pos = [0, 511, 512, slots - 1, slots, 2 * slots + 5, -1]
    b, t = len(pos), max(pos) + 1
    k_all, v_all = rand(b, t, hkv, d, dtype=dtype, seed=3), rand(b, t, hkv, d, dtype=dtype, seed=4)
    kc, vc = S.window_cache(b, hkv, d, window, sinks, dtype)
    kc.fill_(float("nan"))
    vc.fill_(float("nan"))
    at = torch.tensor(pos, device="cuda")
    S.window_cache_fill(k_all, v_all, kc, vc, window, sinks, at.clamp(min=0).to(torch.int32))
    rows = torch.arange(b, device="cuda")
    q = rand(b, hq, d, dtype=dtype, seed=50)
    o = S.window_attention_step(q, k_all[rows, at], v_all[rows, at], kc, vc, at.to(torch.int32), window, sinks)
    within(o, *step_exact(q, k_all, v_all, window, sinks, pos), "o")
    assert (o[-1] == 0).all()
    # one policy alone has the finest ranges
    one = slice(5, 6)
    alone = S.window_attention_step(q[one], k_all[rows, at][one], v_all[rows, at][one], kc[one], vc[one],
                                    at[one].to(torch.int32), window, sinks)
    within(alone, *step_exact(q[one], k_all[one], v_all[one], window, sinks, pos[5:6]), "o alone")


def test_window_step_reads_what_forward_sees():
    """A whole episode token by token gives the rows of one forward call."""
    b, t, hq, hkv, d, window, sinks = 3, 60, 4, 2, 64, 11, 2
    q, k, v = qkv(b, t, hq, hkv, d, BF16)
    want = window_exact(q, k, v, window, sinks)["o"]
    kc, vc = S.window_cache(b, hkv, d, window, sinks, BF16)
    for i in range(t):
        o = S.window_attention_step(q[:, i], k[:, i], v[:, i], kc, vc,
                                    torch.full((b,), i, dtype=torch.int32, device="cuda"), window, sinks)
        within(o, want[0][:, i], want[1][:, i], f"row {i}")


# ---------------------------------------------------------------------------
# Decay attention
# ---------------------------------------------------------------------------
def scan_exact(x, y, z, a, start=None):
    """M_i = a M_{i-1} + y_i^T z_i and x_i M_i, row by row; [b, h, t, .]; `start` is the M before row 0."""
    b, h, t, _ = x.shape
    m = torch.zeros(b, h, x.shape[-1], z.shape[-1], dtype=torch.float64, device="cuda") if start is None else start
    out = torch.zeros(b, h, t, z.shape[-1], dtype=torch.float64, device="cuda")
    for i in range(t):
        m = a[:, None, None] * m + y[:, :, i, :, None] * z[:, :, i, None, :]
        out[:, :, i] = (x[:, :, i, None, :] @ m)[:, :, 0]
    return out, m


def decay_exact(q, k, v, log_decay, state, g=None, dstate=None, scale=None):
    """One batch element of full length: values and magnitudes."""
    c = q.shape[-1] ** -0.5 if scale is None else scale
    a = torch.exp(log_decay.double())
    Q, K, V = (x.double().transpose(1, 2) for x in (q, k, v))
    zero = torch.zeros(q.shape[0], q.shape[2], q.shape[3], v.shape[3], dtype=torch.float64, device="cuda")
    s0 = zero if state is None else state.double()
    ab = lambda *xs: [x.abs() for x in xs]  # noqa: E731
    res = {}

    def put(name, f):
        res[name] = (f(lambda x: x), f(lambda x: x.abs()))

    put("o", lambda m: c * scan_exact(m(Q), m(K), m(V), a, m(s0))[0].transpose(1, 2))
    put("state", lambda m: scan_exact(m(Q), m(K), m(V), a, m(s0))[1])
    if g is not None:
        G = g.double().transpose(1, 2)
        d0 = zero if dstate is None else dstate.double()
        T = lambda x: x.transpose(2, 3)  # noqa: E731
        # the last state's gradient meets the last row undecayed: a start before it, without that row's decay
        t = q.shape[1]
        down = (a[:, None] ** torch.arange(t - 1, -1, -1, device="cuda"))[None, :, :, None]
        put("dq", lambda m: c * scan_exact(m(G), m(V), m(K), a, T(m(s0)).contiguous())[0].transpose(1, 2))
        put("dk", lambda m: (c * scan_exact(m(V).flip(2), m(G).flip(2), m(Q).flip(2), a)[0].flip(2)
                             + down * (m(V) @ T(m(d0)).contiguous())).transpose(1, 2))
        put("dv", lambda m: (c * scan_exact(m(K).flip(2), m(Q).flip(2), m(G).flip(2), a)[0].flip(2)
                             + down * (m(K) @ m(d0))).transpose(1, 2))
        up = (a[:, None] ** torch.arange(1, t + 1, device="cuda"))[None, :, :, None]
        whole = (a ** t)[:, None, None]
        put("dstate", lambda m: c * T(m(Q) * up).contiguous() @ m(G) + whole * m(d0))
    return res


def check_decay(b, t, h, dk, dv, dtype, log_decay=None, lengths=None, with_state=True, with_dstate=True, fused=True, scale=None):
    if fused:
        p = rand(b, t, h, 2 * dk + dv, dtype=dtype, seed=t)
        q, k, v = p[..., :dk], p[..., dk:2 * dk], p[..., 2 * dk:]
    else:
        q, k, v = (rand(b, h, t, d, dtype=dtype, seed=t + i).transpose(1, 2) for i, d in enumerate((dk, dk, dv)))
    if log_decay is None:
        log_decay = torch.log1p(-1.0 / 2.0 ** torch.linspace(1, 9, h, device="cuda"))
    state = rand(b, h, dk, dv, seed=5, scale=3.0) if with_state else None
    dstate = rand(b, h, dk, dv, seed=6) if with_dstate else None
    g = rand(b, t, h, dv, dtype=dtype, seed=8)
    if lengths is not None:
        q, k, v, g = (x.clone() for x in (q, k, v, g))
        for i, n in enumerate(lengths.tolist()):
            for x in (q, k, v, g):
                x[i, n:] = float("nan")
    o, last = S.decay_attention_forward(q, k, v, log_decay, state, lengths, scale)
    grads = S.decay_attention_backward(g, q, k, v, log_decay, state, dstate, lengths, scale)
    got = dict(zip(("o", "state", "dq", "dk", "dv", "dstate"), (o, last) + grads))
    u, tiny = U[dtype], TINY[dtype]
    for i in range(b):
        n = t if lengths is None else int(lengths[i])
        one = lambda x: None if x is None else x[i:i + 1]  # noqa: E731
        want = decay_exact(q[i:i + 1, :n], k[i:i + 1, :n], v[i:i + 1, :n], log_decay, one(state), g[i:i + 1, :n], one(dstate), scale)
        for name, (x, size) in want.items():
            y = got[name][i:i + 1]
            if name in ("state", "dstate"):
                within(y, x, SINGLE * size, name)
                continue
            assert (y[:, n:] == 0).all(), name
            # products of rows and the state are rounded; what is below float16's normal
            # range is off by `tiny` for each of at most 64 rows and 128 columns
            within(y[:, :n], x, u * x.abs() + (u + SINGLE) * size + tiny * 1024, name)


@pytest.mark.parametrize("t", [1, 2, 63, 64, 65, 128, 200])
@pytest.mark.parametrize("dk,dv", [(64, 64), (128, 128), (64, 128), (128, 64), (8, 8), (40, 72)])
def test_decay_lengths_and_dims(t, dk, dv):
    check_decay(2, t, 3, dk, dv, BF16)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("with_state,with_dstate", [(False, False), (True, False), (False, True)])
def test_decay_without_states(dtype, with_state, with_dstate):
    check_decay(2, 130, 2, 64, 64, dtype, with_state=with_state, with_dstate=with_dstate, fused=False)


@pytest.mark.parametrize("dk,dv", [(64, 64), (128, 64)])
def test_decay_segments(dk, dv):
    """Few heads and many rows: cut into segments."""
    check_decay(1, 1100, 2, dk, dv, BF16)
    check_decay(1, 1100, 1, dk, dv, F16, torch.tensor([math.log(0.999)], device="cuda"))


def test_decay_ragged():
    lengths = torch.tensor([300, 0, 1, 64, 65, 299], dtype=torch.int32, device="cuda")
    check_decay(6, 300, 2, 64, 64, BF16, lengths=lengths)
    lengths = torch.tensor([900, 0, 256, 257], dtype=torch.int32, device="cuda")
    check_decay(4, 900, 1, 64, 128, BF16, lengths=lengths)


@pytest.mark.parametrize("t,dk,dv,dtype", [(8192, 64, 64, BF16), (8193, 64, 64, BF16), (8704, 40, 72, F16), (9001, 128, 64, BF16)])
def test_decay_many_segments(t, dk, dv, dtype):
    """64 segments, one more, and numbers of them that eight parts do not share evenly."""
    check_decay(1, t, 1, dk, dv, dtype, torch.tensor([math.log(0.9999)], device="cuda"))
    lengths = torch.tensor([t - 200], dtype=torch.int32, device="cuda")
    check_decay(1, t, 1, dk, dv, dtype, torch.tensor([math.log(0.99)], device="cuda"), lengths=lengths, with_dstate=False)


@pytest.mark.parametrize("t,dk,dv", [(512, 64, 64), (513, 64, 64), (256, 128, 64), (257, 64, 128), (700, 128, 128)])
def test_decay_ragged_segments(t, dk, dv):
    """Around the rows from which sequences are cut: episodes that end before, at and
    behind a segment's first row."""
    lengths = [t, 0, 1, 127, 128, 129, t - 1]
    check_decay(len(lengths), t, 2, dk, dv, BF16, lengths=torch.tensor(lengths, dtype=torch.int32, device="cuda"))


def test_decay_none_and_all():
    """No decay, and one that forgets everything at once."""
    check_decay(1, 150, 2, 64, 64, F16, torch.tensor([0.0, -math.inf], device="cuda"), with_state=False, with_dstate=False)
    check_decay(1, 600, 3, 64, 64, BF16, torch.tensor([0.0, -20.0, -1e-4], device="cuda"))


def test_decay_many_heads():
    check_decay(40, 70, 16, 64, 64, BF16)


def test_decay_scale():
    check_decay(1, 100, 2, 64, 64, BF16, scale=1.0)


def test_decay_without_rows():
    q = torch.empty(2, 0, 3, 64, dtype=BF16, device="cuda")
    state = rand(2, 3, 64, 64, seed=1)
    ld = torch.full((3,), -0.1, device="cuda")
    o, last = S.decay_attention_forward(q, q, q, ld, state)
    assert o.shape == (2, 0, 3, 64) and torch.equal(last, state)
    assert (S.decay_attention_forward(q, q, q, ld)[1] == 0).all()


def test_decay_state_in_place():
    """The state after the rows may replace the one before them, also where a sequence is cut."""
    q, k, v = qkv(1, 1100, 2, 2, 64, BF16, "plain")
    ld = torch.tensor([-0.01, -0.1], device="cuda")
    s = rand(1, 2, 64, 64, seed=2)
    o, last = S.decay_attention_forward(q, k, v, ld, s)
    _, cfg, size = S._decay_setup(q, k, v, ld, None, True, "qds_decay_forward_workspace")
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    o2, s2 = torch.empty_like(o), s.clone()
    assert size > 0 and S.lib().qds_decay_forward(cfg, S._view(q), S._view(k), S._view(v), ld.data_ptr(), s2.data_ptr(),
                                     None, S._view(o2), s2.data_ptr(), ws.data_ptr(), size, S._stream(q)) == S.OK
    assert torch.equal(o, o2) and torch.equal(last, s2)


@pytest.mark.parametrize("dk,dv", [(64, 64), (128, 128), (64, 128), (128, 64), (8, 8), (40, 72)])
@pytest.mark.parametrize("dtype", [BF16, F16])
def test_decay_steps(dk, dv, dtype):
    """An episode token by token, in place and into another state."""
    b, t, h = 3, 12, 2
    q, k, v = (rand(b, t, h, d, dtype=dtype, seed=i) for i, d in enumerate((dk, dk, dv)))
    ld = torch.tensor([-0.5, -math.inf], device="cuda")
    s = rand(b, h, dk, dv, seed=4)
    first = s.clone()
    for i in range(t):
        before = s.clone()
        other = torch.empty_like(s)
        o2, s2 = S.decay_attention_step(q[:, i], k[:, i], v[:, i], ld, before, out_state=other)
        o, s1 = S.decay_attention_step(q[:, i], k[:, i], v[:, i], ld, s)
        assert s1 is s and s2 is other and torch.equal(s, s2) and torch.equal(o, o2)
        want = decay_exact(q[:, :i + 1], k[:, :i + 1], v[:, :i + 1], ld[:1], first) if h == 1 else None
        assert want is None
    for j in range(h):
        one = lambda x: x[:, :, j:j + 1]  # noqa: E731
        if ld[j] == -math.inf:
            eo = dk ** -0.5 * (one(q)[:, -1].double() * one(k)[:, -1].double()).sum(-1, keepdim=True) * one(v)[:, -1].double()
            es = one(k)[:, -1].double()[..., :, None] * one(v)[:, -1].double()[..., None, :]
            so, ss = eo.abs() + dk ** -0.5 * (one(q)[:, -1].double().abs() * one(k)[:, -1].double().abs()).sum(-1, keepdim=True) * one(v)[:, -1].double().abs(), es.abs()
        else:
            want = decay_exact(one(q), one(k), one(v), ld[j:j + 1], first[:, j:j + 1])
            eo, so = want["o"][0][:, -1], want["o"][1][:, -1]
            es, ss = want["state"]
        within(o[:, j:j + 1], eo, U[dtype] * eo.abs() + SINGLE * so + TINY[dtype], "o")
        within(s[:, j:j + 1], es, SINGLE * ss, "state")


def test_decay_gradient_against_differences():
    """As for the window: float16, exact inputs and steps; o is around 3."""
    b, t, h, d = 2, 100, 2, 64
    gen = lambda i: torch.Generator("cuda").manual_seed(i)  # noqa: E731
    q, k, v = ((torch.randint(-32, 33, (b, t, h, d), device="cuda", generator=gen(i)) / 32).to(F16) for i in range(3))
    ld = torch.tensor([-0.05, -0.5], device="cuda")
    g, gs = rand(b, t, h, d, dtype=F16, seed=5), rand(b, h, d, d, seed=6)
    s = rand(b, h, d, d, seed=7)
    xs = [x.clone().requires_grad_() for x in (q, k, v)] + [s.clone().requires_grad_()]
    o, last = S.decay_attention(xs[0], xs[1], xs[2], ld, xs[3], scale=0.125)
    ((o.float() * g.float()).sum() + (last * gs).sum()).backward()
    step = 2.0 ** -3
    for i in range(4):
        if i < 3:
            d_ = (torch.randint(-1, 2, (b, t, h, d), device="cuda", generator=gen(20 + i)) * step).to(F16)
        else:
            d_ = torch.randint(-1, 2, (b, h, d, d), device="cuda", generator=gen(23)).float()

        def loss(sign):
            y = [q, k, v, s]
            y[i] = y[i] + sign * d_
            o, last = S.decay_attention_forward(y[0], y[1], y[2], ld, y[3], scale=0.125)
            return float((o.double() * g).sum() + (last.double() * gs).sum())

        # linear in each input: only roundings are left, o's and those of the gradient's own terms
        got = float((xs[i].grad.double() * d_).sum())
        want = (loss(1) - loss(-1)) / 2
        noise = 2.0 ** -11 * float((o.detach().double() * g).norm())
        size = float((xs[i].grad.double() * d_).norm())
        assert abs(got - want) <= 6 * (noise + 2.0 ** -10 * size), (i, got, want, noise, size)


# ---------------------------------------------------------------------------
# Streams, graphs, arguments
# ---------------------------------------------------------------------------
def calls():
    """One call of each operator on fixed inputs; each returns fresh tensors."""
    x, r, w = norm_inputs(50, 1000, BF16, BF16)
    q, k, v = qkv(2, 300, 4, 2, 64, BF16)
    g = rand(2, 300, 4, 64, dtype=BF16, seed=3)
    p = rand(1, 600, 2, 192, dtype=BF16, seed=4)
    ld = torch.tensor([-0.1, -0.01], device="cuda")
    kc, vc = rand(2, 2, 2003, 64, dtype=BF16, seed=5), rand(2, 2, 2003, 64, dtype=BF16, seed=6)
    pos = torch.tensor([700, 2500], dtype=torch.int32, device="cuda")
    s = rand(1, 2, 64, 64, seed=9)

    def norm():
        y, h, rstd = S.residual_norm_forward(x, r, w)
        return (y, h) + S.residual_norm_backward(x, r, h, rstd, w) + S.residual_norm_fp8(x, r, w)

    def win():
        o, lse = S.window_attention_forward(q, k, v, 50, 3)
        return (o,) + S.window_attention_backward(g, q, k, v, o, lse, 50, 3)

    def step():
        return (S.window_attention_step(q[:, 0], k[:, 0], v[:, 0], kc, vc, pos, 2000, 3),)

    def dec():
        a = p[..., :64], p[..., 64:128], p[..., 128:]
        return S.decay_attention_forward(*a, ld, s) + S.decay_attention_backward(a[0], *a, ld, s, s)

    def dec_step():
        return S.decay_attention_step(p[:, 0, :, :64], p[:, 0, :, 64:128], p[:, 0, :, 128:], ld, s, out_state=torch.empty_like(s))

    return {"norm": norm, "window": win, "window step": step, "decay": dec, "decay step": dec_step}


def same(a, b):
    return all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(a, b))


def test_other_stream():
    """Work goes to the current stream: results there equal those of the default stream."""
    for name, call in calls().items():
        want = call()
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            got = call()
        side.synchronize()
        assert same(got, want), name


def test_graph_replays():
    """Captured once, replayed with the program's own work between the replays."""
    for name, call in calls().items():
        want = [t.clone() for t in call()]
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = call()
        for turn in range(4):
            for t in got:
                t.view(torch.uint8).zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert same(got, want), (name, turn)
            assert same(call(), want), (name, turn)


def test_autograd_matches_the_plain_calls():
    q, k, v = (x.detach().clone().requires_grad_() for x in qkv(2, 100, 4, 2, 64, BF16))
    g = rand(2, 100, 4, 64, dtype=BF16, seed=3)
    S.window_attention(q, k, v, 30, 2).backward(g)
    o, lse = S.window_attention_forward(q.detach(), k.detach(), v.detach(), 30, 2)
    for x, y in zip((q, k, v), S.window_attention_backward(g, q.detach(), k.detach(), v.detach(), o, lse, 30, 2)):
        assert torch.equal(x.grad, y)
    x, r, w = (t.requires_grad_() for t in norm_inputs(20, 256, BF16, BF16))
    y, h = S.residual_norm(x, r, w)
    h.backward(torch.ones_like(h))                     # only the residual is used
    assert (x.grad == 1).all() and (r.grad == 1).all() and w.grad is None


def test_refusals():
    q, k, v = qkv(2, 20, 4, 2, 64, BF16)
    with pytest.raises(ValueError, match="k is"):
        S.window_attention_forward(q, k.float(), v, 4)
    with pytest.raises(ValueError, match="k is"):
        S.window_attention_forward(q, k[:, :10], v, 4)
    with pytest.raises(ValueError, match="multiple"):
        S.window_attention_forward(q[:, :, :3], k, v, 4)
    with pytest.raises(ValueError, match="window"):
        S.window_attention_forward(q, k, v, 0)
    with pytest.raises(ValueError, match="too large"):
        S.window_attention_forward(q, k, v, (1 << 32) + 4)
    with pytest.raises(ValueError, match="lengths"):
        S.window_attention_forward(q, k, v, 4, lengths=torch.tensor([3, 4], device="cuda"))
    with pytest.raises(ValueError, match="lengths is on"):
        S.window_attention_forward(q, k, v, 4, lengths=torch.tensor([3, 4], dtype=torch.int32))
    with pytest.raises(S.SeqError) as e:
        S.window_attention_forward(*qkv(2, 20, 4, 2, 136, BF16), 4)
    assert e.value.status == S.ERR_UNSUPPORTED
    with pytest.raises(S.SeqError) as e:
        S.window_attention_forward(*(x.float() for x in (q, k, v)), 4)
    assert e.value.status == S.ERR_UNSUPPORTED
    with pytest.raises(S.SeqError) as e:
        S.window_attention_forward(q, k, v, 4, scale=-1.0)
    assert e.value.status == S.ERR_INVALID_ARG
    kc, vc = S.window_cache(2, 2, 64, 8, 1, BF16)
    pos = torch.zeros(2, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError, match="k_cache"):
        S.window_attention_step(q[:, 0], k[:, 0], v[:, 0], kc[:, :, :8], vc, pos, 8, 1)
    with pytest.raises(ValueError, match="pos"):
        S.window_attention_step(q[:, 0], k[:, 0], v[:, 0], kc, vc, pos.long(), 8, 1)
    with pytest.raises(ValueError, match="contiguous"):
        S.window_attention_step(q[:, 0], k[:, 0], v[:, 0], kc.transpose(2, 3).contiguous().transpose(2, 3), vc, pos, 8, 1)
    ld = torch.zeros(4, device="cuda")
    with pytest.raises(ValueError, match="log_decay"):
        S.decay_attention_forward(q, q, q, ld[:3])
    with pytest.raises(ValueError, match="state"):
        S.decay_attention_forward(q, q, q, ld, torch.zeros(2, 4, 64, 32, device="cuda"))
    x, r, w = norm_inputs(4, 100, BF16, BF16)
    with pytest.raises(ValueError, match="residual"):
        S.residual_norm_forward(x, r[:2], w)
    with pytest.raises(ValueError, match="weight"):
        S.residual_norm_forward(x, r, w.half())
    with pytest.raises(ValueError, match="group"):
        S.residual_norm_fp8(x, r, w, group=128)
    with pytest.raises(ValueError, match="float32, bfloat16 or float16"):
        S.residual_norm_forward(x.double(), r.double(), w.double())
