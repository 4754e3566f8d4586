"""The selective block's operators on the GPU against their definitions in 64 bits.

Tolerances are bounds worked out from the kernels' roundings, element by element: the result
is rounded once to its type (u = eps / 2: 2^-8 bfloat16, 2^-11 float16, 2^-24 float32), all else
is float32, whose share is a number of roundings times 2^-24 times the sum of the magnitudes
of the terms (from the same definition on absolute values).  The numbers of roundings are
counted at each test.
"""
import pytest

torch = pytest.importorskip("torch")

from helpers import block_definitions as D  # noqa: E402
from paper_2202_01258_amd import seq as S  # noqa: E402

pytestmark = pytest.mark.gpu

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
TYPES = [BF16, F16, F32]
U = {t: torch.finfo(t).eps / 2 for t in TYPES}
TINY = {BF16: 0.0, F16: 2.0 ** -25, F32: 0.0}      # half of the least float16 above 0
E32 = 2.0 ** -24
FLUSH = 2.0 ** -120                                 # numbers below float32's normal range may be 0


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def rand(*shape, dtype=F32, seed=0, scale=1.0):
    g = torch.Generator()
    g.manual_seed(seed * 1000003 + sum(shape))
    return (torch.randn(*shape, generator=g) * scale).to(dtype).cuda()


def wide(t):
    return None if t is None else t.double().cpu()


def within(got, pair, roundings, what, flush=FLUSH):
    want, mag = pair
    assert got.shape == want.shape, (what, got.shape, want.shape)
    got = got.detach()
    u, tiny = (U[got.dtype], TINY[got.dtype])
    bound = u * want.abs() + (1 + u) * roundings * E32 * mag + tiny + flush
    err = (got.double().cpu() - want).abs()
    bad = ~(err <= bound)
    assert not bad.any(), (f"{what}: {int(bad.sum())} of {bad.numel()} outside, worst by "
                           f"{float((err / bound)[bad].max()):.3g} times, first at {bad.nonzero()[0].tolist()}")


def ends_of(lengths, batch, rows):
    return [rows] * batch if lengths is None else [min(max(n, 0), rows) for n in lengths]


def as_lengths(lengths):
    return None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")


def layout(t, how):
    """The same values in another layout; what lies between them is not a number."""
    if how == "plain":
        return t
    nan = float("nan")
    if how == "slice":                              # columns of a wider tensor, rows at odd places
        big = torch.full((*t.shape[:-1], t.shape[-1] + 5), nan, dtype=t.dtype, device=t.device)
        big[..., 3:3 + t.shape[-1]] = t
        return big[..., 3:3 + t.shape[-1]]
    if how == "rows first":                         # [rows, batch, width]
        return t.transpose(0, 1).contiguous().transpose(0, 1)
    assert how == "columns apart"
    return t.transpose(-1, -2).contiguous().transpose(-1, -2)


LAYOUTS = ["slice", "rows first", "columns apart"]


# ---------------------------------------------------------------------------
# Short causal convolution
# ---------------------------------------------------------------------------
def check_conv(batch, rows, width, taps, dtype, wdtype=F32, act=True, lengths=None, bias=True, state=True, how="plain",
               seed=1):
    x, w = rand(batch, rows, width, dtype=dtype, seed=seed), rand(taps, width, dtype=wdtype, seed=seed + 1, scale=taps ** -0.5)
    b = rand(width, dtype=wdtype, seed=seed + 2, scale=0.3) if bias else None
    s = rand(batch, taps - 1, width, dtype=dtype, seed=seed + 3) if state else None
    dy, dlast = rand(batch, rows, width, dtype=dtype, seed=seed + 4), rand(batch, taps - 1, width, dtype=dtype, seed=seed + 5)
    ends = ends_of(lengths, batch, rows)
    want = D.conv(wide(x), wide(w), wide(b) if bias else torch.zeros(width).double(),
                  wide(s) if state else torch.zeros(batch, taps - 1, width).double(), ends, act, wide(dy), wide(dlast))
    for i, n in enumerate(ends):                    # nothing behind a length is read
        x[i, n:] = float("nan")
        dy[i, n:] = float("nan")
    x, dy = layout(x, how), layout(dy, how)
    kw = dict(bias=b, state=s, lengths=as_lengths(lengths), silu=act)
    y, last = S.causal_conv_forward(x, w, **kw)
    # taps fmas, then the exponential, reciprocal and products of silu: 12 at most
    within(y, want["y"], taps + 12, "y")
    assert torch.equal(last.double().cpu(), want["last"][0])
    dx, dw, db, dstate = S.causal_conv_backward(dy, x, w, dlast=dlast, **kw)
    # g: taps + 20; dx: taps more and the last state's; sums over rows: one each at most
    rows_in = sum(ends)
    within(dx, want["dx"], 2 * taps + 24, "dx")
    within(dstate, want["dstate"], 2 * taps + 24, "dstate")
    within(dw, want["dw"], taps + 24 + rows_in, "dw")
    if bias:
        within(db, want["db"], taps + 24 + rows_in, "db")
    else:
        assert db is None
    for i, n in enumerate(ends):
        assert not y[i, n:].any() and not dx[i, n:].any()
    return y, last


@pytest.mark.parametrize("batch,rows,width", [(1, 1, 1), (2, 5, 3), (3, 37, 20), (2, 130, 77), (1, 300, 256), (4, 2, 64),
                                              (2, 70, 1030), (70, 9, 5)])
@pytest.mark.parametrize("taps,dtype", [(4, BF16), (3, F16), (4, F32), (1, BF16), (8, F32), (2, F16)])
def test_conv_sizes(batch, rows, width, taps, dtype):
    check_conv(batch, rows, width, taps, dtype)


@pytest.mark.parametrize("taps", [1, 2, 3, 4, 5, 6, 7, 8])
@pytest.mark.parametrize("act", [True, False])
def test_conv_taps(taps, act):
    check_conv(2, 41, 22, taps, BF16, act=act, lengths=[41, 3])
    check_conv(2, 41, 3, taps, F16, act=act, lengths=[40, 1])


@pytest.mark.parametrize("dtype,wdtype", [(BF16, BF16), (F16, F16), (F32, F32), (BF16, F32)])
def test_conv_lengths(dtype, wdtype):
    check_conv(7, 66, 40, 4, dtype, wdtype, lengths=[66, 0, 1, 2, 3, 65, 32])
    check_conv(3, 66, 40, 4, dtype, wdtype, lengths=[1000, -5, 64])


@pytest.mark.parametrize("how", LAYOUTS)
@pytest.mark.parametrize("width", [16, 33])
def test_conv_layouts(how, width):
    check_conv(3, 20, width, 4, BF16, how=how, lengths=[20, 7, 11])


@pytest.mark.parametrize("bias,state", [(False, True), (True, False), (False, False)])
def test_conv_without(bias, state):
    check_conv(2, 20, 24, 4, F32, bias=bias, state=state)


def test_conv_without_rows():
    """No rows: states go through, the sums are 0."""
    x, w = torch.empty(3, 0, 10, device="cuda"), rand(4, 10)
    state = rand(3, 3, 10, seed=3)
    y, last = S.causal_conv_forward(x, w, state=state)
    assert y.shape == x.shape and torch.equal(last, state)
    dx, dw, db, dstate = S.causal_conv_backward(x, x, w, bias=w[0], state=state, dlast=state)
    assert dx.shape == x.shape and torch.equal(dstate, state) and not dw.any() and not db.any()
    e = torch.empty(0, 5, 10, device="cuda")
    y, last = S.causal_conv_forward(e, w)
    assert y.shape == e.shape and last.shape == (0, 3, 10)
    assert not S.causal_conv_backward(e, e, w)[1].any()


def test_conv_broadcast_batch():
    """One episode seen by a whole batch: strides of 0."""
    x = rand(1, 30, 24, dtype=BF16).expand(5, 30, 24)
    w = rand(4, 24, seed=2)
    y, last = S.causal_conv_forward(x, w)
    want, wlast = S.causal_conv_forward(x.contiguous(), w)
    assert torch.equal(y, want) and torch.equal(last, wlast)
    got, full = S.causal_conv_backward(x, x, w), S.causal_conv_backward(x.contiguous(), x.contiguous(), w)
    assert all(torch.equal(g, f) for g, f in zip((got[0], got[1], got[3]), (full[0], full[1], full[3])))


@pytest.mark.parametrize("taps,width,dtype", [(4, 64, BF16), (3, 7, F16), (8, 33, F32), (1, 5, BF16), (2, 2, F32), (4, 4098, BF16)])
def test_conv_steps(taps, width, dtype):
    """Row by row, in place and into another state: the rows of one forward call."""
    x, w, b = rand(3, 9, width, dtype=dtype), rand(taps, width, seed=2), rand(width, seed=3)
    first = rand(3, taps - 1, width, dtype=dtype, seed=4)
    want, wlast = S.causal_conv_forward(x, w, b, first)
    state, other = first.clone(), first.clone()
    for t in range(9):
        y, got = S.causal_conv_step(layout(x, "slice")[:, t], w, b, state)
        assert got is state
        assert torch.equal(y, want[:, t])
        y2, other = S.causal_conv_step(x[:, t], w, b, other, out_state=torch.empty_like(other))
        assert torch.equal(y2, y)
    assert torch.equal(state, wlast) and torch.equal(other, wlast)


def test_conv_in_parts():
    """An episode in two calls that pass the state on, forward and backward."""
    x, w, b = rand(2, 50, 24), rand(4, 24, seed=2), rand(24, seed=3)
    dy = rand(2, 50, 24, seed=4)
    y, last = S.causal_conv_forward(x, w, b)
    dx, dw, db, _ = S.causal_conv_backward(dy, x, w, b)
    for cut in (1, 2, 33):
        y1, s1 = S.causal_conv_forward(x[:, :cut], w, b)
        y2, s2 = S.causal_conv_forward(x[:, cut:], w, b, s1)
        assert torch.equal(torch.cat([y1, y2], 1), y) and torch.equal(s2, last)
        dx2, dw2, db2, ds = S.causal_conv_backward(dy[:, cut:], x[:, cut:], w, b, s1)
        dx1, dw1, db1, _ = S.causal_conv_backward(dy[:, :cut], x[:, :cut], w, b, dlast=ds)
        # the state's gradient is a partial sum, rounded: the order of 4 fmas
        assert (torch.cat([dx1, dx2], 1) - dx).abs().max() <= 64 * E32 * dx.abs().max()
        assert (dw1 + dw2 - dw).abs().max() <= 200 * E32 * (x.abs().max() * dy.abs().sum((0, 1)).max())
        assert (db1 + db2 - db).abs().max() <= 200 * E32 * 1.1 * dy.abs().sum((0, 1)).max()


# ---------------------------------------------------------------------------
# Selective state space scan
# ---------------------------------------------------------------------------
def scan_inputs(batch, rows, width, states, dtype, seed=1):
    g = torch.Generator()
    g.manual_seed(seed)
    step = torch.exp(torch.rand(width, generator=g) * 4.6 - 6.9)
    bc = rand(batch, rows, 2 * states, dtype=dtype, seed=seed)
    rate = torch.arange(1, states + 1) * torch.exp(0.3 * torch.randn(width, states, generator=g))
    return dict(u=rand(batch, rows, width, dtype=dtype, seed=seed + 1), delta=rand(batch, rows, width, dtype=dtype, seed=seed + 2),
                a=-rate.cuda(), b=bc[..., :states], c=bc[..., states:], skip=rand(width, seed=seed + 3),
                gate=rand(batch, rows, width, dtype=dtype, seed=seed + 4), bias=torch.log(torch.expm1(step)).cuda(),
                state=rand(batch, width, states, seed=seed + 5)), dict(
        do=rand(batch, rows, width, dtype=dtype, seed=seed + 6), dlast=rand(batch, width, states, seed=seed + 7))


def check_scan(batch, rows, width, states, dtype, lengths=None, without=(), how="plain", seed=1, backward=True):
    s, g = scan_inputs(batch, rows, width, states, dtype, seed)
    ends = ends_of(lengths, batch, rows)
    w = {k: wide(v) for k, v in s.items()}
    if "skip" in without:
        w["skip"] = torch.zeros_like(w["skip"])
    if "bias" in without:
        w["bias"] = torch.zeros_like(w["bias"])
    if "state" in without:
        w["state"] = torch.zeros_like(w["state"])
    if "gate" in without:
        w["gate"] = torch.full_like(w["gate"], 1.2784645427610738)        # silu is 1 here
    wdlast = torch.zeros_like(w["state"]) if "dlast" in without else wide(g["dlast"])
    want, top = D.scan(**w, ends=ends, do=wide(g["do"]), dlast=wdlast)
    for i, n in enumerate(ends):                     # nothing behind a length is read
        for t in (s["u"], s["delta"], s["b"], s["c"], s["gate"], g["do"]):
            t[i, n:] = float("nan")
    s = {k: layout(v, how) if k in ("u", "delta", "b", "c", "gate") else v for k, v in s.items()}
    do, dlast = layout(g["do"], how), g["dlast"]
    for k in without:
        s[k] = None
    if "dlast" in without:
        dlast = None
    s.pop("dlast", None)
    state = s.pop("state")
    x = [s.pop(k) for k in ("u", "delta", "a", "b", "c")]
    kw = dict(**s, lengths=as_lengths(lengths))
    o, last, marks = S.selective_scan_forward(*x, state=state, keep=True, **kw)
    # Each row adds the roundings of a decay (its exponent's, 4 dt |a| in all, and the exponential's),
    # of an input (8 for the step, 2 products) and of two fmas; a segment's start as many once more.
    # Behind that, the sum over states, skip and gate.
    per_row = 16 + 6 * top
    path = per_row * (max(ends, default=0) + 2)
    within(o, want["o"], path + states + 16, "o")
    within(last, want["last"], path, "last")
    for i, n in enumerate(ends):
        assert not o[i, n:].any()
    again = S.selective_scan_forward(*x, state=state, **kw)
    assert torch.equal(again[0], o) and torch.equal(again[1], last) and again[2] is None
    if not backward:
        return
    got = dict(zip(("du", "ddelta", "da", "db", "dc", "dskip", "dgate", "dbias", "dstate"),
                   S.selective_scan_backward(do, *x, marks, dlast=dlast, **kw)))
    # a gradient is a product of what comes from before and from behind, twice the path; then
    # sums over states, columns, rows and the batch
    sums = {"du": states, "ddelta": states, "da": sum(ends), "db": width, "dc": width, "dskip": sum(ends), "dgate": states,
            "dbias": states + sum(ends), "dstate": 0}
    for name, v in got.items():
        if (name == "dskip" and "skip" in without) or (name == "dgate" and "gate" in without) or (
                name == "dbias" and "bias" in without):
            assert v is None
            continue
        within(v, want[name], 2 * path + 32 + sums[name], name)
    for i, n in enumerate(ends):
        for name in ("du", "ddelta", "db", "dc"):
            assert not got[name][i, n:].any()


@pytest.mark.parametrize("batch,rows,width", [(1, 1, 1), (2, 5, 3), (3, 37, 20), (1, 130, 77), (4, 2, 64), (2, 33, 200),
                                              (1, 17, 130)])
@pytest.mark.parametrize("states,dtype", [(16, BF16), (4, F16), (13, F32), (1, F32), (8, BF16), (32, F16), (24, F32)])
def test_scan_sizes(batch, rows, width, states, dtype):
    check_scan(batch, rows, width, states, dtype)


@pytest.mark.parametrize("states", [2, 3, 5, 7, 9, 15, 17, 31, 32])
def test_scan_states(states):
    check_scan(2, 19, 21, states, F32, lengths=[19, 16])


@pytest.mark.parametrize("states", [4, 8, 16, 32])
@pytest.mark.parametrize("dtype", TYPES)
def test_scan_lengths(states, dtype):
    check_scan(9, 50, 18, states, dtype, lengths=[50, 0, 1, 15, 16, 17, 49, 100, -3])


@pytest.mark.parametrize("rows", [64, 65, 128, 300, 331])
@pytest.mark.parametrize("states", [4, 16, 32])
def test_scan_segments(rows, states):
    """Few columns: an episode is cut into segments that run side by side."""
    check_scan(1, rows, 16, states, F32)
    check_scan(3, rows, 9, states, BF16, lengths=[rows, 63, 0])
    check_scan(3, rows, 9, states, F16, lengths=[rows - 1, 64, 65])


@pytest.mark.parametrize("states", [4, 13, 16, 32])
def test_scan_many_pieces(states):
    """More pieces than the main pass follows by itself: a scan over them joins them."""
    check_scan(1, 1057, 7, states, F32)
    check_scan(2, 1400, 70, states, BF16, lengths=[1400, 1060])
    check_scan(3, 1100, 5, states, F16, lengths=[0, 1, 1099])


@pytest.mark.parametrize("states", [4, 16, 32])
def test_scan_pieces_of_segments(states):
    """Several pieces for each segment of the gradients' main pass, which ends inside them."""
    check_scan(16, 300, 256, states, BF16, lengths=[300, 0, 1, 31, 32, 33, 63, 64, 65, 95, 96, 97, 128, 200, 299, 300])


@pytest.mark.parametrize("how", LAYOUTS)
def test_scan_layouts(how):
    check_scan(3, 40, 17, 16, BF16, how=how, lengths=[40, 7, 31])


@pytest.mark.parametrize("without", [("skip",), ("gate",), ("bias",), ("state",), ("dlast",),
                                     ("skip", "gate", "bias", "state", "dlast")])
def test_scan_without(without):
    check_scan(2, 70, 20, 16, F32, without=without)


def test_scan_many_episodes():
    """More segments than workgroups that go through them: shares of da come from several."""
    check_scan(1100, 3, 8, 4, F32)
    check_scan(40, 5, 1030, 4, BF16, lengths=[5, 4, 0, 1] * 10)


def test_scan_without_rows():
    """No rows: states and their gradients go through, the sums are 0."""
    s, g = scan_inputs(3, 0, 10, 16, F32)
    x = [s[k] for k in ("u", "delta", "a", "b", "c")]
    kw = dict(skip=s["skip"], gate=s["gate"], bias=s["bias"])
    o, last, marks = S.selective_scan_forward(*x, state=s["state"], keep=True, **kw)
    assert o.shape == s["u"].shape and torch.equal(last, s["state"])
    du, ddelta, da, db, dc, dskip, dgate, dbias, dstate = S.selective_scan_backward(g["do"], *x, marks, dlast=g["dlast"], **kw)
    assert torch.equal(dstate, g["dlast"]) and not da.any() and not dskip.any() and not dbias.any()
    s, g = scan_inputs(0, 5, 10, 16, F32)
    x = [s[k] for k in ("u", "delta", "a", "b", "c")]
    o, last, marks = S.selective_scan_forward(*x, state=s["state"], keep=True, **kw | {"gate": s["gate"]})
    assert last.shape == (0, 10, 16)
    assert not S.selective_scan_backward(g["do"], *x, marks, dlast=g["dlast"], **kw | {"gate": s["gate"]})[2].any()


@pytest.mark.parametrize("states,dtype", [(16, BF16), (13, F32), (4, F16), (32, BF16), (1, F32)])
@pytest.mark.parametrize("width", [64, 37])
def test_scan_steps(states, dtype, width):
    """Row by row, in place and into another state: the rows of one forward call, whose sums over
    states are in another order."""
    s, _ = scan_inputs(3, 9, width, states, dtype)
    want, top = D.scan(**{k: wide(v) for k, v in s.items()}, ends=[9] * 3)
    a, skip, bias = s["a"], s["skip"], s["bias"]
    state, other, out = s["state"].clone(), s["state"].clone(), []
    for t in range(9):
        row = [layout(s[k], "slice")[:, t] for k in ("u", "delta", "b", "c", "gate")]
        o, got = S.selective_scan_step(row[0], row[1], a, row[2], row[3], state, skip, row[4], bias)
        assert got is state
        o2, other = S.selective_scan_step(row[0], row[1], a, row[2], row[3], other, skip, row[4], bias,
                                          out_state=torch.empty_like(other))
        assert torch.equal(o, o2)
        out.append(o)
    path = (16 + 6 * top) * 11
    within(torch.stack(out, 1), want["o"], path + states + 16, "o")
    within(state, want["last"], path, "last")
    assert torch.equal(state, other)


def test_scan_step_without():
    s, _ = scan_inputs(2, 1, 20, 16, F32)
    state = s["state"].clone()
    o, _ = S.selective_scan_step(s["u"][:, 0], s["delta"][:, 0], s["a"], s["b"][:, 0], s["c"][:, 0], state)
    want, last, _ = S.selective_scan_forward(s["u"], s["delta"], s["a"], s["b"], s["c"], state=s["state"])
    assert torch.allclose(o, want[:, 0], rtol=64 * E32, atol=64 * E32) and torch.allclose(state, last, rtol=64 * E32, atol=64 * E32)


def test_scan_not_finite():
    """A number that is not finite stays in its column and episode, and reaches only the rows
    behind it; one of b or c reaches its row's columns.  A rate of minus infinity forgets all."""
    s, _ = scan_inputs(2, 150, 40, 16, F32)
    x = lambda t: [t[k] for k in ("u", "delta", "a", "b", "c")]  # noqa: E731
    kw = dict(skip=s["skip"], gate=s["gate"], bias=s["bias"], state=s["state"])
    want, last, _ = S.selective_scan_forward(*x(s), **kw)
    bad = dict(s, u=s["u"].clone())
    bad["u"][1, 70, 5] = float("nan")
    o, l2, _ = S.selective_scan_forward(*x(bad), **kw)
    hit = torch.zeros_like(o, dtype=torch.bool)
    hit[1, 70:, 5] = True
    assert torch.equal(o.isnan(), hit) and torch.equal(o[~hit], want[~hit])
    bad = dict(s, c=s["c"].clone())
    bad["c"][0, 3, 2] = float("inf")
    o, l2, _ = S.selective_scan_forward(*x(bad), **kw)
    hit = torch.zeros_like(o, dtype=torch.bool)
    hit[0, 3] = True
    assert torch.equal(~o.isfinite(), hit) and torch.equal(o[~hit], want[~hit]) and torch.equal(l2, last)
    forget = dict(s, a=torch.full_like(s["a"], -float("inf")))
    lengths = torch.tensor([150, 65], dtype=torch.int32, device="cuda")
    o, l2, _ = S.selective_scan_forward(*x(forget), lengths=lengths, **kw)
    assert o.isfinite().all() and l2.isfinite().all()
    dt = torch.logaddexp(s["delta"].double() + s["bias"].double(), torch.zeros((), device="cuda").double())
    for i, n in enumerate((150, 65)):
        only = (dt[i, n - 1] * s["u"][i, n - 1].double())[:, None] * s["b"][i, n - 1].double()
        assert (l2[i].double() - only).abs().max() <= 16 * E32 * only.abs().max()


@pytest.mark.parametrize("scale", [30.0, 100.0, 1000.0])
def test_scan_steps_of_any_size(scale):
    """Steps from e^-1000 (which is 0) to 1000."""
    s, g = scan_inputs(1, 20, 16, 4, F32)
    s["delta"] = s["delta"] * scale
    s["bias"] = None
    x = [s[k] for k in ("u", "delta", "a", "b", "c")]
    want, top = D.scan(**{k: wide(v) for k, v in s.items() if k != "bias"}, bias=torch.zeros(16).double(), ends=[20],
                       do=wide(g["do"]), dlast=wide(g["dlast"]))
    # A step or slope below 2^-126 is 0 in float32 (slope 7.8e-39 at raw -87.75, scale 30, where
    # ddelta is 2.3e-36): what it multiplies is lost, 2^-126 times the factor's magnitude, up to
    # 415, 1918 and 19414 at the three scales
    slope = torch.sigmoid(wide(s["delta"]))
    factor = float((want["ddelta"][1] / slope)[slope > 0].max())
    flush = FLUSH + 2.0 ** -126 * factor
    o, last, marks = S.selective_scan_forward(*x, skip=s["skip"], gate=s["gate"], state=s["state"], keep=True)
    within(o, want["o"], (16 + 6 * top) * 22 + 20, "o", flush)
    within(last, want["last"], (16 + 6 * top) * 22, "last", flush)
    got = S.selective_scan_backward(g["do"], *x, marks, skip=s["skip"], gate=s["gate"], dlast=g["dlast"])
    for name, v in zip(("du", "ddelta", "da", "db", "dc", "dskip", "dgate"), got):
        within(v, want[name], (16 + 6 * top) * 44 + 80, name, flush)


def test_scan_in_parts():
    """Two calls that pass the state on give the outputs of one, and the gradients."""
    s, g = scan_inputs(2, 100, 24, 16, F32)
    names = ("u", "delta", "a", "b", "c")
    part = lambda rows: [s[k] if k == "a" else s[k][:, rows] for k in names]  # noqa: E731
    kw = lambda rows: dict(skip=s["skip"], gate=s["gate"][:, rows], bias=s["bias"])  # noqa: E731
    want, top = D.scan(**{k: wide(v) for k, v in s.items()}, ends=[100, 100], do=wide(g["do"]), dlast=wide(g["dlast"]))
    one, two = slice(0, 37), slice(37, 100)
    o1, mid, m1 = S.selective_scan_forward(*part(one), state=s["state"], keep=True, **kw(one))
    o2, last, m2 = S.selective_scan_forward(*part(two), state=mid, keep=True, **kw(two))
    path = (16 + 6 * top) * 104
    within(torch.cat([o1, o2], 1), want["o"], path + 32, "o")
    within(last, want["last"], path, "last")
    g2 = S.selective_scan_backward(g["do"][:, two], *part(two), m2, dlast=g["dlast"], **kw(two))
    g1 = S.selective_scan_backward(g["do"][:, one], *part(one), m1, dlast=g2[-1], **kw(one))
    within(g1[-1], want["dstate"], 2 * path + 32, "dstate")
    for i, name in ((0, "du"), (1, "ddelta"), (3, "db"), (4, "dc"), (6, "dgate")):
        within(torch.cat([g1[i], g2[i]], 1), want[name], 2 * path + 80, name)
    for i, name in ((2, "da"), (5, "dskip"), (7, "dbias")):
        within(g1[i] + g2[i], want[name], 2 * path + 300, name)


def test_scan_gradient_against_differences():
    """The kernel's own outputs at two points along a direction, against its gradient: what the
    definition says the difference misses is added, and the outputs' roundings over the step."""
    s, g = scan_inputs(2, 70, 9, 5, F32)
    order = ("u", "delta", "a", "b", "c", "skip", "gate", "bias", "state")
    way = {k: rand(*s[k].shape, seed=50 + i) * (0.05 if k == "a" else 1.0) for i, k in enumerate(order)}
    eps = 2.0 ** -7

    def at(e):
        return {k: s[k] + e * way[k] for k in order}

    def loss(t):
        o, last, _ = S.selective_scan_forward(*[t[k] for k in order[:5]], t["skip"], t["gate"], t["bias"], t["state"])
        return float((o.double() * g["do"].double()).sum() + (last.double() * g["dlast"].double()).sum())

    def exact(t):
        out, top = D.scan(**{k: wide(v) for k, v in t.items()}, ends=[70, 70])
        do, dl = wide(g["do"]), wide(g["dlast"])
        value = float((out["o"][0] * do).sum() + (out["last"][0] * dl).sum())
        mag = float((out["o"][1] * do.abs()).sum() + (out["last"][1] * dl.abs()).sum())
        return value, (16 + 6 * top) * 72 * E32 * mag

    marks = S.selective_scan_forward(*[s[k] for k in order[:5]], s["skip"], s["gate"], s["bias"], s["state"], keep=True)[2]
    got = dict(zip(("u", "delta", "a", "b", "c", "skip", "gate", "bias", "state"), S.selective_scan_backward(
        g["do"], *[s[k] for k in order[:5]], marks, s["skip"], s["gate"], s["bias"], g["dlast"])))
    along = sum(float((got[k].double() * way[k].double()).sum()) for k in order)
    full, _ = D.scan(**{k: wide(v) for k, v in s.items()}, ends=[70, 70], do=wide(g["do"]), dlast=wide(g["dlast"]))
    names = dict(zip(order, ("du", "ddelta", "da", "db", "dc", "dskip", "dgate", "dbias", "dstate")))
    true = sum(float((full[names[k]][0] * wide(way[k])).sum()) for k in order)
    (up, eu), (down, ed) = exact(at(eps)), exact(at(-eps))
    missed = abs((up - down) / (2 * eps) - true)
    difference = (loss(at(eps)) - loss(at(-eps))) / (2 * eps)
    assert abs(difference - along) <= missed + (eu + ed) / (2 * eps) + 1e-3 * abs(true)
    assert abs(along - true) <= 1e-4 * abs(true) + 1e-3


# ---------------------------------------------------------------------------
# Norms after and before a block
# ---------------------------------------------------------------------------
EPS = 1e-6
BRANCH_SHAPES = [(1, 1), (5, 7), (3, 64), (9, 128), (1, 512), (17, 520), (6, 777), (4, 1000), (3, 1024), (5, 2048), (3, 2056),
                 (2, 4096), (3, 5000), (2, 8192), (2, 9001), (600, 40)]
# a sum over a row: at most 80 roundings on the way of a term (chains of 16 and a tree of ten, or
# chains of 40 and a tree), a norm's factor 8, the gate 10; two norms and two sums follow each other
ROUNDINGS = 400


@pytest.mark.parametrize("rows,width", BRANCH_SHAPES)
@pytest.mark.parametrize("dtype,wdtype", [(BF16, BF16), (F16, F32), (F32, F32)])
def test_branch(rows, width, dtype, wdtype, gate=True, scale=0.75, how="plain"):
    x, g, r = (rand(rows, width, dtype=dtype, seed=i, scale=2.0 ** (i - 1)) for i in range(3))
    w1, w2 = ((1 + 0.2 * rand(width, seed=i)).to(wdtype) for i in (5, 6))
    dy, dh = rand(rows, width, dtype=dtype, seed=7), rand(rows, width, dtype=dtype, seed=8)
    flat = torch.full((rows, width), 1.2784645427610738).double()                      # silu is 1 here
    want = D.branch(wide(x), wide(g) if gate else flat, wide(r), wide(w1), wide(w2), scale, EPS, wide(dy), wide(dh))
    x, g, r, dy, dh = (layout(t, how) for t in (x, g, r, dy, dh))
    g = g if gate else None
    y, h, rstds = S.branch_norm_forward(x, g, r, w1, w2, scale, EPS)
    within(y, want["y"], ROUNDINGS, "y")
    within(h, want["h"], ROUNDINGS, "h")
    within(rstds[0], want["rx"], ROUNDINGS, "rx")
    within(rstds[1], want["rh"], ROUNDINGS, "rh")
    dx, dg, dr, dw1, dw2 = S.branch_norm_backward(dy, dh, x, g, r, rstds, w1, w2, scale)
    within(dx, want["dx"], 3 * ROUNDINGS, "dx")
    within(dr, want["dresidual"], 2 * ROUNDINGS, "dresidual")
    within(dw1, want["dw1"], 3 * ROUNDINGS + rows, "dw1")
    within(dw2, want["dw2"], 2 * ROUNDINGS + rows, "dw2")
    if gate:
        within(dg, want["dgate"], 2 * ROUNDINGS, "dgate")
    else:
        assert dg is None


@pytest.mark.parametrize("width", [128, 520, 9001])
def test_branch_without_gate(width):
    test_branch(5, width, F32, F32, gate=False)
    test_branch(5, width, BF16, F32, gate=False, scale=-1.0)


@pytest.mark.parametrize("how", ["slice", "columns apart"])
@pytest.mark.parametrize("width", [128, 1024, 9216])
def test_branch_layouts(how, width):
    test_branch(6, width, BF16, F32, how=how)


def test_branch_without_rows_and_without_dh():
    x, w = torch.empty(0, 3, 40, device="cuda"), rand(40)
    y, h, rstds = S.branch_norm_forward(x, x, x, w, w)
    assert y.shape == x.shape and rstds.shape == (2, 0, 3)
    got = S.branch_norm_backward(x, None, x, x, x, rstds, w, w)
    assert not got[3].any() and not got[4].any()
    x, g, r, dy = (rand(2, 3, 40, seed=i) for i in range(4))
    rstds = S.branch_norm_forward(x, g, r, w, w)[2]
    a = S.branch_norm_backward(dy, None, x, g, r, rstds, w, w)
    b = S.branch_norm_backward(dy, torch.zeros_like(dy), x, g, r, rstds, w, w)
    assert all(torch.equal(p, q) for p, q in zip(a, b))


def test_branch_special_rows():
    """Rows of zeros are zeros; a row with a number that is not finite stays by itself."""
    x, g, r = (rand(5, 200, seed=i) for i in range(3))
    w = torch.ones(200, device="cuda")
    x[1], r[1] = 0, 0
    x[3, 7] = float("nan")
    y, h, _ = S.branch_norm_forward(x, g, r, w, w, 1.0, EPS)
    assert not y[1].any() and not h[1].any()
    assert y[3].isnan().all() and y[[0, 2, 4]].isfinite().all()


# ---------------------------------------------------------------------------
# Dropout
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("shape", [(1,), (7,), (8,), (9,), (3, 5), (2, 3, 64), (257, 33), (1, 4099)])
@pytest.mark.parametrize("dtype", TYPES)
def test_dropout(shape, dtype):
    seed, step, site, p = 0x123456789ABCDEF, (5 << 32) + 77, 9, 0.3
    rng = S.dropout_rng(seed, step)
    x, r = rand(*shape, dtype=dtype, seed=1), rand(*shape, dtype=dtype, seed=2)
    n = x.numel()
    limit = int(p * 65536 + 0.5)
    keep = torch.tensor([d >= limit for d in D.draws(range(n), seed, step, site)]).view(shape)
    up = 65536 / (65536 - limit)
    kept = torch.where(keep, wide(x) * up, torch.zeros(()).double())
    for residual in (None, r):
        y = S.dropout_forward(x, rng, p, site, residual)
        base = torch.zeros_like(kept) if residual is None else wide(residual)
        within(y, (base + kept, base.abs() + kept.abs()), 4, "y")
        if residual is None:
            assert torch.equal((y == 0).cpu(), ~keep | (wide(x) == 0))
    within(S.dropout_backward(x, rng, p, site), (kept, kept.abs()), 4, "dx")


def test_dropout_layouts_and_extremes():
    rng = S.dropout_rng(-3, 1)
    x = rand(20, 30, dtype=BF16)
    want = S.dropout_forward(x, rng, 0.5, residual=x)
    for how in ("slice", "columns apart"):
        assert torch.equal(S.dropout_forward(layout(x, how), rng, 0.5, residual=layout(x, how)), want)
    assert torch.equal(S.dropout_forward(x, rng, 0.0), x)
    x[3, 4] = float("inf")
    y = S.dropout_forward(x, rng, 0.999)
    assert y[3, 4] == 0 or y[3, 4] == float("inf")                # dropped, not 0 times infinity
    assert S.dropout_forward(torch.empty(0, 5, device="cuda"), rng, 0.5).shape == (0, 5)


def test_dropout_draws_are_independent():
    """Shares of kept elements, and of those kept at both of two seeds, steps or sites: within six
    standard deviations."""
    n, p = 1 << 20, 0.25
    x = torch.ones(n, device="cuda")
    base = S.dropout_forward(x, S.dropout_rng(1, 0), p) > 0
    sigma = (n * p * (1 - p)) ** 0.5
    assert abs(int(base.sum()) - n * (1 - p)) < 6 * sigma
    for seed, step, site in ((2, 0, 0), (1, 1, 0), (1, 0, 1), (1 + (1 << 32), 0, 0), (1, 1 << 32, 0)):
        other = S.dropout_forward(x, S.dropout_rng(seed, step), p, site) > 0
        q = (1 - p) ** 2
        assert abs(int((base & other).sum()) - n * q) < 6 * (n * q * (1 - q)) ** 0.5
    for lag in (1, 2, 8, 64, 1000):
        q = (1 - p) ** 2
        assert abs(int((base[lag:] & base[:-lag]).sum()) - (n - lag) * q) < 6 * 2 * (n * q * (1 - q)) ** 0.5


# ---------------------------------------------------------------------------
# Streams, graphs, autograd, arguments
# ---------------------------------------------------------------------------
def calls():
    """Each operator's calls on inputs of their own: {name: function that returns tensors}."""
    x, w = rand(3, 200, 40, dtype=BF16), rand(4, 40, seed=1)
    lengths = torch.tensor([200, 0, 131], dtype=torch.int32, device="cuda")
    s, g = scan_inputs(3, 200, 40, 16, BF16)
    sx = [s[k] for k in ("u", "delta", "a", "b", "c")]
    kw = dict(skip=s["skip"], gate=s["gate"], bias=s["bias"], lengths=lengths)
    state, conv_state = torch.empty_like(s["state"]), rand(3, 3, 40, dtype=BF16, seed=6)
    b = [rand(3, 200, 40, dtype=BF16, seed=10 + i) for i in range(5)]
    rng = S.dropout_rng(4, 2)

    def conv():
        y, last = S.causal_conv_forward(x, w, lengths=lengths)
        dx, dw, _, ds = S.causal_conv_backward(y, x, w, lengths=lengths)
        return y, last, dx, dw, ds

    def scan():
        o, last, marks = S.selective_scan_forward(*sx, state=s["state"], keep=True, **kw)
        return (o, last) + S.selective_scan_backward(g["do"], *sx, marks, dlast=g["dlast"], **kw)

    def step():
        y, cs = S.causal_conv_step(x[:, 0], w, None, conv_state, out_state=torch.empty_like(conv_state))
        o, _ = S.selective_scan_step(sx[0][:, 0], sx[1][:, 0], sx[2], sx[3][:, 0], sx[4][:, 0], s["state"], out_state=state)
        return y, cs, o, state

    def branch():
        y, h, rstds = S.branch_norm_forward(b[0], b[1], b[2], w[0], w[1], 0.5)
        return (y, h) + S.branch_norm_backward(b[3], b[4], b[0], b[1], b[2], rstds, w[0], w[1], 0.5)

    def dropout():
        return S.dropout_forward(x, rng, 0.2, 3, x), S.dropout_backward(x, rng, 0.2, 3)

    return {"conv": conv, "scan": scan, "step": step, "branch": branch, "dropout": dropout}


def same(got, want):
    return all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(got, want))


def test_same_from_call_to_call():
    for name, call in calls().items():
        want = [t.clone() for t in call()]
        for _ in range(3):
            assert same(call(), want), name


def test_other_stream():
    """Work goes to the current stream: results on a side stream, and on two at once, are the same."""
    todo = calls()
    want = {name: [t.clone() for t in call()] for name, call in todo.items()}
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for name, call in todo.items():
        if name == "step":
            continue                                  # writes one state: not for two streams
        got = []
        for st in streams:
            with torch.cuda.stream(st):
                got.append(call())
        torch.cuda.synchronize()
        assert same(got[0], want[name]) and same(got[1], want[name]), name


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


def test_captured_dropout_draws_anew():
    """A replay reads the step: after the program changed it, another mask, that of the eager call."""
    rng, x = S.dropout_rng(8, 0), torch.ones(4096, device="cuda")
    S.dropout_forward(x, rng, 0.5)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = S.dropout_forward(x, rng, 0.5)
    seen = []
    for step in range(4):
        rng[1] = step
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, S.dropout_forward(x, rng, 0.5))
        seen.append(y.clone())
    assert not any(torch.equal(seen[i], seen[j]) for i in range(4) for j in range(i))


def test_autograd_matches_the_plain_calls():
    leaf = lambda t: t.detach().clone().requires_grad_()  # noqa: E731
    x, w, bias, st = leaf(rand(2, 40, 24)), leaf(rand(4, 24, seed=1)), leaf(rand(24, seed=2)), leaf(rand(2, 3, 24, seed=3))
    lengths = torch.tensor([40, 11], dtype=torch.int32, device="cuda")
    dy, dlast = rand(2, 40, 24, seed=4), rand(2, 3, 24, seed=5)
    y, last = S.causal_conv(x, w, bias, st, lengths)
    got = torch.autograd.grad([y, last], [x, w, bias, st], [dy, dlast])
    assert same(got, S.causal_conv_backward(dy, x, w, bias, st, dlast, lengths))
    (gx,) = torch.autograd.grad(S.causal_conv(x, w, bias, st, lengths)[1], [x], dlast)          # the last state alone
    assert torch.equal(gx, S.causal_conv_backward(torch.zeros_like(dy), x, w, bias, st, dlast, lengths)[0])

    s, g = scan_inputs(2, 40, 24, 16, F32)
    t = {k: leaf(v) for k, v in s.items()}
    names = ("u", "delta", "a", "b", "c", "skip", "gate", "bias")
    o, last = S.selective_scan(*[t[k] for k in names], t["state"], lengths)
    got = torch.autograd.grad([o, last], [t[k] for k in names] + [t["state"]], [g["do"], g["dlast"]])
    marks = S.selective_scan_forward(*[s[k] for k in names], s["state"], lengths, keep=True)[2]
    want = S.selective_scan_backward(g["do"], *[s[k] for k in names[:5]], marks, *[s[k] for k in names[5:]], g["dlast"], lengths)
    assert same(got, want)
    with torch.no_grad():
        assert same(S.selective_scan(*[t[k] for k in names], t["state"], lengths), (o.detach(), last.detach()))
    o, _ = S.selective_scan(*[t[k] for k in names[:5]])
    assert len(torch.autograd.grad(o.sum(), [t[k] for k in names[:5]])) == 5

    x, gate, r = (leaf(rand(2, 7, 24, seed=i)) for i in range(3))
    w1, w2 = leaf(rand(24, seed=5)), leaf(rand(24, seed=6))
    dy, dh = rand(2, 7, 24, seed=8), rand(2, 7, 24, seed=9)
    y, h = S.branch_norm(x, gate, r, w1, w2, 0.5)
    got = torch.autograd.grad([y, h], [x, gate, r, w1, w2], [dy, dh])
    rstds = S.branch_norm_forward(x, gate, r, w1, w2, 0.5)[2]
    assert same(got, S.branch_norm_backward(dy, dh, x, gate, r, rstds, w1, w2, 0.5))
    got = torch.autograd.grad(S.branch_norm(x, None, r, w1, w2)[1], [x, r], dh)                 # h alone
    assert torch.equal(got[1], dh)

    rng = S.dropout_rng(3)
    y = S.dropout(x, rng, 0.4, 2, r)
    gx, gr = torch.autograd.grad(y, [x, r], dy)
    assert torch.equal(gx, S.dropout_backward(dy, rng, 0.4, 2)) and torch.equal(gr, dy)
    y = S.dropout(x, rng, 0.4)
    rng[1] += 1
    with pytest.raises(RuntimeError, match="modified"):
        y.sum().backward()


def test_refusals():
    x, w, n = rand(2, 10, 24, dtype=BF16), rand(4, 24), rand(2, 10, 16, dtype=BF16)
    a = -rand(24, 16).abs()
    bad = [
        lambda: S.causal_conv_forward(x[0], w), lambda: S.causal_conv_forward(x, w[:, :8]), lambda: S.causal_conv_forward(x, w.half()),
        lambda: S.causal_conv_forward(x, torch.cat([w, w, w])), lambda: S.causal_conv_forward(x, w, bias=w[0].bfloat16()),
        lambda: S.causal_conv_forward(x, w, state=rand(2, 4, 24, dtype=BF16)), lambda: S.causal_conv_forward(x.long(), w),
        lambda: S.causal_conv_forward(x, w, lengths=torch.ones(2, device="cuda")),
        lambda: S.causal_conv_backward(x[:, :5], x, w), lambda: S.causal_conv_backward(x, x, w, dlast=rand(2, 3, 24)),
        lambda: S.causal_conv_step(x[:, 0], w, None, rand(2, 24, 3, dtype=BF16).transpose(1, 2)),
        lambda: S.causal_conv_step(x, w, None, x),
        lambda: S.selective_scan_forward(x, x[:, :5], a, n, n), lambda: S.selective_scan_forward(x, x, a.half(), n, n),
        lambda: S.selective_scan_forward(x, x, a[:, :8], n, n), lambda: S.selective_scan_forward(x, x, rand(24, 33), n, n),
        lambda: S.selective_scan_forward(x, x, a, n, n[:1]), lambda: S.selective_scan_forward(x, x, a, n, n, gate=n),
        lambda: S.selective_scan_forward(x, x, a, n, n, skip=w[0].bfloat16()),
        lambda: S.selective_scan_forward(x, x, a, n, n, bias=w),
        lambda: S.selective_scan_forward(x, x, a, n, n, state=rand(2, 24, 15)),
        lambda: S.selective_scan_backward(x, x, x, a, n, n, torch.empty(16, dtype=torch.uint8, device="cuda")),
        lambda: S.selective_scan_step(x[:, 0], x[:, 0], a, n[:, 0], n[:, 0], rand(2, 24, 16).bfloat16()),
        lambda: S.branch_norm_forward(x, x[:1], x, w[0], w[0]), lambda: S.branch_norm_forward(x, None, x.float(), w[0], w[0]),
        lambda: S.branch_norm_forward(x, None, x, w[0], w[0].bfloat16()), lambda: S.branch_norm_forward(x, None, x, w, w),
        lambda: S.branch_norm_backward(x, None, x, None, x, rand(2, 2, 9), w[0], w[0]),
        lambda: S.dropout_forward(x, S.dropout_rng(1), 1.0), lambda: S.dropout_forward(x, S.dropout_rng(1), -0.1),
        lambda: S.dropout_forward(x, S.dropout_rng(1), 1 - 2.0 ** -18), lambda: S.dropout_forward(x, S.dropout_rng(1), 0.5, -1),
        lambda: S.dropout_forward(x, S.dropout_rng(1).int(), 0.5), lambda: S.dropout_forward(x, S.dropout_rng(1), 0.5, residual=n),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            pytest.fail(f"call {i} was not refused")
    for scale in (float("nan"), float("inf")):
        with pytest.raises(S.SeqError):
            S.branch_norm_forward(x, None, x, w[0], w[0], residual_scale=scale)


def test_beyond_31_bits():
    """Episodes, rows and states that start more than 2^31 elements into their tensors."""
    big = torch.zeros((1 << 31) + (1 << 20), dtype=BF16, device="cuda")
    far = big.as_strided((2, 80, 24), (1 << 31, 24, 1))
    far.copy_(rand(2, 80, 24, dtype=BF16))
    near, w = far.contiguous(), rand(4, 24, seed=2)
    assert same(S.causal_conv_forward(far, w), S.causal_conv_forward(near, w))
    got, want = S.causal_conv_backward(far, far, w), S.causal_conv_backward(near, near, w)
    assert all(torch.equal(got[i], want[i]) for i in (0, 1, 3))
    s, g = scan_inputs(2, 80, 24, 16, BF16)
    n = (s["a"], s["b"], s["c"])
    o, last, marks = S.selective_scan_forward(far, far, *n, gate=far, keep=True)
    wo, wlast, wmarks = S.selective_scan_forward(near, near, *n, gate=near, keep=True)
    assert torch.equal(o, wo) and torch.equal(last, wlast)
    got = S.selective_scan_backward(far, far, far, *n, marks, gate=far)
    want = S.selective_scan_backward(near, near, near, *n, wmarks, gate=near)
    assert all(torch.equal(got[i], want[i]) for i in (0, 1, 2, 3, 4, 6, 8))
    # rows 2^23 elements apart and more: the scan's are copied, the convolution takes them
    for apart in ((1 << 23) - 8, 1 << 23, (1 << 24) + 3):
        rows = big.as_strided((1, 100, 24), (0, apart, 1))
        rows.copy_(near[:1, :50].repeat(1, 2, 1))
        assert same(S.causal_conv_forward(rows, w), S.causal_conv_forward(rows.contiguous(), w))
        m = [t[:1, :50].repeat(1, 2, 1) for t in (s["b"], s["c"])]
        assert same(S.selective_scan_forward(rows, rows, s["a"], *m)[:2],
                    S.selective_scan_forward(rows.contiguous(), rows.contiguous(), s["a"], *m)[:2])
    x = big[: 1 << 31].view(1 << 17, 1 << 14)
    rng = S.dropout_rng(1)
    x.fill_(1.0)
    y = S.dropout_forward(x, rng, 0.5)
    tail = range((1 << 31) - 4096, 1 << 31)
    keep = torch.tensor([d >= 32768 for d in D.draws(tail, 1, 0, 0)])
    assert torch.equal((y.view(-1)[-4096:] > 0).cpu(), keep)
    del y
    x[:, :64] = 0.5
    view = x[:, 64:64 + 700]                           # rows 2^14 apart over 2^31 elements
    w = torch.ones(700, device="cuda")
    y, h, rstds = S.branch_norm_forward(view, view, view, w, w)
    assert torch.equal(y[:8], y[-8:]) and torch.equal(h[:8], h[-8:])
    got = S.branch_norm_backward(y, h, view, view, view, rstds, w, w)
    assert torch.equal(got[0][:8], got[0][-8:]) and torch.equal(got[2][:8], got[2][-8:])
