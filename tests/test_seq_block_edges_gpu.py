"""The selective block's operators on the GPU where they can go wrong beyond ordinary sizes and numbers."""
import pytest

torch = pytest.importorskip("torch")

from helpers import block_definitions as D  # noqa: E402
from paper_2202_01258_amd import seq as S  # noqa: E402
from test_seq_block_gpu import BF16, E32, F16, F32, TYPES, rand, same, scan_inputs, wide, within  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


NAMES = ("u", "delta", "a", "b", "c")


def args(s):
    """The first arguments of the scan's calls, and the others."""
    return [s[k] for k in NAMES], {k: v for k, v in s.items() if k not in (*NAMES, "state")}


def test_scan_of_more_than_2_to_the_23_columns():
    """16384 short episodes of 513 columns: outputs and gradients of some of them against the
    definition, all of them against those of two calls with half of the batch, whose shares of the sums over the
    batch are added in another order: 3 * 16384 terms, each side."""
    batch, rows, width = 16384, 3, 513
    s, g = scan_inputs(batch, rows, width, 4, BF16)
    x, kw = args(s)
    o, last, marks = S.selective_scan_forward(*x, state=s["state"], keep=True, **kw)
    got = S.selective_scan_backward(g["do"], *x, marks, dlast=g["dlast"], **kw)
    some = [0, 8191, 8192, batch - 1]
    part = lambda t: wide(t[some])  # noqa: E731
    want, top = D.scan(**{k: part(v) if k in ("u", "delta", "b", "c", "gate", "state") else wide(v) for k, v in s.items()},
                       ends=[rows] * 4, do=part(g["do"]), dlast=part(g["dlast"]))
    path = (16 + 6 * top) * (rows + 2)
    within(o[some], want["o"], path + 20, "o")
    within(last[some], want["last"], path, "last")
    sums = {0: ("du", 4), 1: ("ddelta", 4), 3: ("db", width), 4: ("dc", width), 6: ("dgate", 4), 8: ("dstate", 0)}
    for i, (name, n) in sums.items():
        within(got[i][some], want[name], 2 * path + 32 + n, name)
    ends = []
    for half in (slice(0, batch // 2), slice(batch // 2, batch)):
        hx = [t if k == "a" else t[half] for k, t in zip(NAMES, x)]
        hkw = dict(kw, gate=kw["gate"][half])
        ho, hlast, hmarks = S.selective_scan_forward(*hx, state=s["state"][half], keep=True, **hkw)
        assert torch.equal(ho, o[half]) and torch.equal(hlast, last[half])
        hgot = S.selective_scan_backward(g["do"][half], *hx, hmarks, dlast=g["dlast"][half], **hkw)
        for i in sums:
            assert torch.equal(hgot[i], got[i][half]), sums[i][0]
        ends.append(hgot)
    terms = 2 * batch * rows * E32
    gate = kw["gate"].double()
    mag = (g["do"].double() * gate * torch.sigmoid(gate) * x[0].double()).abs().sum((0, 1))
    assert ((ends[0][5] + ends[1][5] - got[5]).abs() <= 1.001 * terms * mag).all()
    assert ((ends[0][7] + ends[1][7] - got[7]).abs() <= 1.01 * terms * got[1].double().abs().sum((0, 1))).all()
