"""The selective block's operators on the CPU: struct layouts, refusals before any GPU work, the
binding's checks, scratch memory, and the definitions that the GPU tests compare with."""
import ctypes as C
import os
import shutil
import subprocess

import pytest

torch = pytest.importorskip("torch")

from helpers import block_definitions as D  # noqa: E402
from paper_2202_01258_amd import seq as S  # noqa: E402

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 1 << 20                                       # a pointer that nothing may follow


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(S.LIB_PATH):
        pytest.skip("libqdseq.so not built")
    return S.lib()


def rows(p=P, strides=(64, 64)):
    return S.QdsRows(p, *strides)


NONE = S.QdsRows(None, 0, 0)


def make(kind, fields, over):
    f = dict(fields)
    f.update(over)
    return kind(*[f[n] for n, _ in kind._fields_])


def conv(**over):
    return make(S.QdsConvConfig, dict(abi_version=S.ABI_VERSION, dtype=S.BF16, weight_dtype=S.F32, batch=2, length=100,
                                      width=64, taps=4, silu=1), over)


def scan(**over):
    return make(S.QdsScanConfig, dict(abi_version=S.ABI_VERSION, dtype=S.BF16, batch=2, length=1000, width=64,
                                      states=16), over)


def branch(**over):
    return make(S.QdsBranchConfig, dict(abi_version=S.ABI_VERSION, dtype=S.BF16, weight_dtype=S.F32, width=64, rows=10,
                                        eps=1e-6, residual_scale=1.0), over)


def dropout(**over):
    return make(S.QdsDropoutConfig, dict(abi_version=S.ABI_VERSION, dtype=S.BF16, elements=100, threshold=100, site=0),
                over)


def bytes_of(fn, cfg):
    n = C.c_uint64()
    return fn(C.byref(cfg), C.byref(n)), n.value


def test_struct_layouts_match_the_header(lib, tmp_path):
    if shutil.which("gcc") is None:
        pytest.skip("gcc not available")
    kinds = [("qds_rows", S.QdsRows, "stride"), ("qds_conv_config", S.QdsConvConfig, "silu"),
             ("qds_scan_config", S.QdsScanConfig, "states"), ("qds_branch_config", S.QdsBranchConfig, "residual_scale"),
             ("qds_dropout_config", S.QdsDropoutConfig, "site")]
    src = tmp_path / "sz.c"
    lines = "".join(f'printf("%zu %zu ", sizeof({n}), offsetof({n}, {f}));' for n, _, f in kinds)
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "qd_seq.h"\nint main(void){' + lines + "return 0;}\n")
    exe = tmp_path / "sz"
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    got = [int(t) for t in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()]
    want = []
    for _, kind, last in kinds:
        want += [C.sizeof(kind), getattr(kind, "stride_b" if last == "stride" else last).offset]
    assert got == want


# -- refusals
CONV_BAD = [(dict(abi_version=0), S.ERR_INVALID_ARG), (dict(dtype=3), S.ERR_INVALID_ARG), (dict(dtype=-1), S.ERR_INVALID_ARG),
            (dict(weight_dtype=S.F16), S.ERR_INVALID_ARG), (dict(batch=-1), S.ERR_INVALID_ARG),
            (dict(length=-1), S.ERR_INVALID_ARG), (dict(length=1 << 30), S.ERR_INVALID_ARG), (dict(width=0), S.ERR_INVALID_ARG),
            (dict(width=(1 << 20) + 1), S.ERR_INVALID_ARG), (dict(taps=0), S.ERR_INVALID_ARG), (dict(taps=9), S.ERR_INVALID_ARG),
            (dict(silu=2), S.ERR_INVALID_ARG), (dict(batch=1 << 28, length=1000), S.ERR_UNSUPPORTED)]


@pytest.mark.parametrize("over,status", CONV_BAD)
def test_conv_refusals(lib, over, status):
    c = conv(**over)
    assert lib.qds_causal_conv(C.byref(c), rows(), P, P, P, None, rows(2 * P), P + 4096, None) == status
    assert bytes_of(lib.qds_causal_conv_backward_workspace, c)[0] == status
    if "length" not in over:
        assert lib.qds_causal_conv_step(C.byref(c), rows(), P, P, P, rows(), P, None) == status


def test_conv_refuses_pointers(lib):
    c = conv()
    ok = [C.byref(c), rows(), P, P, P, None, rows(2 * P), P + 4096, None]
    for i, bad in [(0, None), (1, NONE), (2, None), (6, NONE), (6, rows()), (7, P)]:     # y is not x, one state not the other
        a = list(ok)
        a[i] = bad
        assert lib.qds_causal_conv(*a) == S.ERR_INVALID_ARG
    st, need = bytes_of(lib.qds_causal_conv_backward_workspace, c)
    assert st == S.OK and need >= 5 * 64 * 4
    ok = [C.byref(c), rows(), rows(), P, P, P, P, None, rows(), P, P, P + 4096, P, need, None]
    for i, bad in [(1, NONE), (2, NONE), (3, None), (8, NONE), (9, None), (11, P), (12, None), (12, P + 64)]:
        a = list(ok)
        a[i] = bad
        assert lib.qds_causal_conv_backward(*a) == S.ERR_INVALID_ARG
    ok[13] = need - 1
    assert lib.qds_causal_conv_backward(*ok) == S.ERR_WORKSPACE_TOO_SMALL
    ok = [C.byref(c), rows(), P, P, P, rows(), P, None]
    for i, bad in [(1, NONE), (2, None), (4, None), (5, NONE), (6, None)]:
        a = list(ok)
        a[i] = bad
        assert lib.qds_causal_conv_step(*a) == S.ERR_INVALID_ARG


SCAN_BAD = [(dict(abi_version=7), S.ERR_INVALID_ARG), (dict(dtype=5), S.ERR_INVALID_ARG), (dict(batch=-2), S.ERR_INVALID_ARG),
            (dict(length=-1), S.ERR_INVALID_ARG), (dict(length=1 << 30), S.ERR_INVALID_ARG), (dict(width=0), S.ERR_INVALID_ARG),
            (dict(width=1 << 21), S.ERR_INVALID_ARG), (dict(states=0), S.ERR_INVALID_ARG), (dict(states=33), S.ERR_UNSUPPORTED),
            (dict(batch=1 << 26, length=1), S.ERR_UNSUPPORTED)]


@pytest.mark.parametrize("over,status", SCAN_BAD)
def test_scan_refusals(lib, over, status):
    c, r = scan(**over), rows()
    assert bytes_of(lib.qds_selective_scan_workspace, c)[0] == status
    assert bytes_of(lib.qds_selective_scan_backward_workspace, c)[0] == status
    assert lib.qds_selective_scan(C.byref(c), r, r, P, r, r, P, r, P, P, None, P, P, P, P, 1 << 40, None) == status
    assert lib.qds_selective_scan_backward(C.byref(c), r, r, r, P, r, r, P, r, P, P, P, None, P, P, P, P, P, P, P, P, P, P,
                                           1 << 40, None) == status
    if "length" not in over:
        assert lib.qds_selective_scan_step(C.byref(c), r, r, P, r, r, P, r, P, P, P, P, None) == status


def test_scan_refuses_pointers(lib):
    c, r = scan(batch=1, width=16), rows()
    st, need = bytes_of(lib.qds_selective_scan_workspace, c)
    assert st == S.OK and need > 0                    # few columns: their rows are cut into segments
    ok = [C.byref(c), r, r, P, r, r, P, r, P, P, None, P, P + 4096, P, P, need, None]
    far, back = rows(strides=(1, 1 << 23)), rows(strides=(1, -64))
    for i, bad in [(0, None), (1, NONE), (2, NONE), (3, None), (4, NONE), (5, NONE), (11, None), (12, P), (13, P + 64), (14, None),
                   (14, P + 128)]:
        a = list(ok)
        a[i] = bad
        assert lib.qds_selective_scan(*a) == S.ERR_INVALID_ARG, i
    for i in (1, 2, 4, 5, 7):
        for bad in (far, back):
            a = list(ok)
            a[i] = bad
            assert lib.qds_selective_scan(*a) == S.ERR_UNSUPPORTED, i
    ok[15] = need - 1
    assert lib.qds_selective_scan(*ok) == S.ERR_WORKSPACE_TOO_SMALL
    st, need = bytes_of(lib.qds_selective_scan_backward_workspace, c)
    ok = [C.byref(c), r, r, r, P, r, r, P, r, P, P, P, None, P, P, P, P, P, P, P, P, P + 4096, P, need, None]
    for i, bad in [(1, NONE), (2, NONE), (3, NONE), (4, None), (5, NONE), (6, NONE), (10, None), (10, P + 16), (13, None),
                   (14, None), (15, None), (16, None), (17, None), (19, None), (21, P), (22, None), (22, P + 4)]:
        a = list(ok)
        a[i] = bad
        assert lib.qds_selective_scan_backward(*a) == S.ERR_INVALID_ARG, i
    for i in (1, 2, 3, 5, 6, 8):
        for bad in (far, back):
            a = list(ok)
            a[i] = bad
            assert lib.qds_selective_scan_backward(*a) == S.ERR_UNSUPPORTED, i
    ok[23] = need - 1
    assert lib.qds_selective_scan_backward(*ok) == S.ERR_WORKSPACE_TOO_SMALL
    ok = [C.byref(c), r, r, P, r, r, P, r, P, P, P, P, None]
    for i, bad in [(1, NONE), (2, NONE), (3, None), (4, NONE), (5, NONE), (9, None), (10, None), (11, None)]:
        a = list(ok)
        a[i] = bad
        assert lib.qds_selective_scan_step(*a) == S.ERR_INVALID_ARG, i


@pytest.mark.parametrize("over", [dict(abi_version=2), dict(dtype=3), dict(weight_dtype=S.F16), dict(width=0),
                                  dict(width=(1 << 20) + 1), dict(rows=-1), dict(rows=1 << 31), dict(eps=-1.0),
                                  dict(eps=float("nan")), dict(residual_scale=float("nan")),
                                  dict(residual_scale=float("inf"))])
def test_branch_refusals(lib, over):
    c = branch(**over)
    assert lib.qds_branch_norm(C.byref(c), P, 64, P, 64, P, 64, P, P, P, P, P, None) == S.ERR_INVALID_ARG
    assert bytes_of(lib.qds_branch_norm_backward_workspace, c)[0] == S.ERR_INVALID_ARG


def test_branch_refuses_pointers(lib):
    c = branch()
    for missing in (1, 5, 7, 8, 9, 10, 11):
        a = [C.byref(c), P, 64, P, 64, P, 64, P, P, P, P, P, None]
        a[missing] = None
        assert lib.qds_branch_norm(*a) == S.ERR_INVALID_ARG
    st, need = bytes_of(lib.qds_branch_norm_backward_workspace, c)
    assert st == S.OK and need == 10 * 2 * 64 * 4
    ok = [C.byref(c), P, 64, P, 64, P, 64, P, 64, P, 64, P, P, P, P, P, P, P, P, P, need, None]
    for missing in (1, 5, 9, 11, 12, 13, 14, 15, 16, 17, 18, 19):
        a = list(ok)
        a[missing] = None
        assert lib.qds_branch_norm_backward(*a) == S.ERR_INVALID_ARG, missing
    ok[20] = need - 1
    assert lib.qds_branch_norm_backward(*ok) == S.ERR_WORKSPACE_TOO_SMALL
    ok[20], ok[19] = need, P + 64
    assert lib.qds_branch_norm_backward(*ok) == S.ERR_INVALID_ARG


def test_dropout_refusals(lib):
    for over in (dict(abi_version=2), dict(dtype=3), dict(elements=-1), dict(elements=(1 << 34) + 1), dict(threshold=65536)):
        assert lib.qds_dropout(C.byref(dropout(**over)), P, P, P, P, None) == S.ERR_INVALID_ARG, over
    for missing in (0, 1, 3, 4):
        a = [C.byref(dropout()), P, P, P, P, None]
        a[missing] = None
        assert lib.qds_dropout(*a) == S.ERR_INVALID_ARG


def test_empty_calls_launch_nothing(lib):
    assert lib.qds_causal_conv(C.byref(conv(batch=0)), NONE, P, None, None, None, NONE, None, None) == S.OK
    assert lib.qds_causal_conv_step(C.byref(conv(batch=0)), NONE, P, None, None, NONE, None, None) == S.OK
    assert lib.qds_selective_scan(C.byref(scan(batch=0)), NONE, NONE, P, NONE, NONE, None, NONE, None, None, None, None, None,
                                  None, None, 0, None) == S.OK
    assert lib.qds_selective_scan_step(C.byref(scan(batch=0)), NONE, NONE, P, NONE, NONE, None, NONE, None, None, None, None,
                                       None) == S.OK
    assert lib.qds_branch_norm(C.byref(branch(rows=0)), *[None, 0] * 3, *[None] * 6) == S.OK
    assert lib.qds_dropout(C.byref(dropout(elements=0)), None, None, None, None, None) == S.OK


def test_scratch_memory_stays_small(lib):
    """Shares of db and dc are what grows: 2 * 16 floats for 128 columns of a row, against the
    14 bytes of each of its numbers that the pass moves."""
    c = scan(batch=32, length=1000, width=1024)
    need = bytes_of(lib.qds_selective_scan_backward_workspace, c)[1]
    assert need < 0.3 * 14 * 32 * 1000 * 1024
    # one mark, [columns][states] fp32, for 8 rows
    assert bytes_of(lib.qds_selective_scan_marks, c)[1] == 32 * 125 * 1024 * 16 * 4
    assert bytes_of(lib.qds_causal_conv_backward_workspace, conv(batch=32, length=1000, width=1024))[1] <= 2048 * 5 * 128 * 4


# -- the binding's checks
def test_binding_needs_a_gpu():
    x, w = torch.zeros(2, 5, 8), torch.zeros(4, 8)
    a, n = torch.zeros(8, 4), torch.zeros(2, 5, 4)
    for call in (lambda: S.causal_conv_forward(x, w), lambda: S.causal_conv(x, w),
                 lambda: S.causal_conv_step(x[:, 0], w, None, torch.zeros(2, 3, 8)),
                 lambda: S.selective_scan_forward(x, x, a, n, n), lambda: S.selective_scan(x, x, a, n, n),
                 lambda: S.selective_scan_step(x[:, 0], x[:, 0], a, n[:, 0], n[:, 0], torch.zeros(2, 8, 4)),
                 lambda: S.branch_norm_forward(x, x, x, w[0], w[0]), lambda: S.branch_norm(x, None, x, w[0], w[0]),
                 lambda: S.dropout_forward(x, torch.zeros(2, dtype=torch.int64), 0.5)):
        with pytest.raises(RuntimeError, match="GPU"):
            call()


# -- the definitions
def test_philox_known_answers():
    """The published known answers of Philox4x32-10."""
    assert D.philox((0, 0, 0, 0), (0, 0)) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    ones = 0xFFFFFFFF
    assert D.philox((ones,) * 4, (ones,) * 2) == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]
    assert D.philox((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0)) == [
        0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1]


def test_definitions_by_hand():
    """One column, one state, three rows, in closed form."""
    t = lambda *v: torch.tensor(v, dtype=torch.float64)  # noqa: E731
    x = t(1.0, 2.0, 3.0).view(1, 3, 1)
    out = D.conv(x, t(0.5, 2.0).view(2, 1), t(0.25), t(7.0).view(1, 1, 1), [3], False)
    assert out["y"][0].flatten().tolist() == [0.25 + 3.5 + 2, 0.25 + 0.5 + 4, 0.25 + 1 + 6] and out["last"][0].item() == 3
    raw = torch.log(torch.expm1(t(0.5)))
    out, _ = D.scan(x, torch.zeros(1, 3, 1).double(), t(-2.0).view(1, 1), t(1.0, 1.0, 2.0).view(1, 3, 1),
                    t(1.0, 1.0, 1.0).view(1, 3, 1), t(10.0), t(0.0, 0.0, 0.0).view(1, 3, 1), raw, t(4.0).view(1, 1, 1), [2])
    e = torch.exp(t(-1.0))
    h = e * 4 + 0.5
    h = e * h + 1.0
    assert abs(out["last"][0].item() - h.item()) < 1e-14 and out["o"][0].abs().max() == 0    # silu(0) = 0
