"""libqdseq.so and its binding on the CPU: exported symbols, struct layouts,
refusals before any GPU work, and the index arithmetic of the ring cache and of
the backward pass's work items, replayed on the host."""
import ctypes as C
import os
import re
import shutil
import subprocess

import pytest

from paper_2202_01258_amd import seq as S

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(S.LIB_PATH):
        pytest.skip("libqdseq.so not built")
    return S.lib()


def test_exports_every_declared_symbol(lib):
    header = open(os.path.join(ROOT, "include", "qd_seq.h")).read()
    declared = set(re.findall(r"^\s*(?:const char\*|qds_status)\s+(qds_\w+)\s*\(", header, re.M))
    assert declared == set(S.EXPORTS)
    for name in declared:
        assert hasattr(lib, name)


def test_no_kernel_needs_scratch_memory(lib):
    key = b".private_segment_fixed_size"          # a msgpack map entry: key, then an integer
    data = open(S.LIB_PATH, "rb").read()
    sizes = [data[m.end()] for m in re.finditer(re.escape(key), data)]
    assert len(sizes) > 60                        # every kernel instance
    assert all(size == 0 for size in sizes), sizes


def test_struct_layouts_match_the_header(lib, tmp_path):
    if shutil.which("gcc") is None:
        pytest.skip("gcc not available")
    src = tmp_path / "sz.c"
    src.write_text(
        '#include <stdio.h>\n#include <stddef.h>\n#include "qd_seq.h"\n'
        'int main(void){printf("%zu %zu %zu %zu %zu %zu %zu\\n", sizeof(qds_view), sizeof(qds_norm_config), '
        'offsetof(qds_norm_config, group), sizeof(qds_window_config), offsetof(qds_window_config, scale), '
        'sizeof(qds_decay_config), offsetof(qds_decay_config, scale)); return 0;}\n')
    exe = tmp_path / "sz"
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    got = [int(t) for t in subprocess.run([str(exe)], capture_output=True, text=True,
                                          check=True).stdout.split()]
    assert got == [C.sizeof(S.QdsView), C.sizeof(S.QdsNormConfig), S.QdsNormConfig.group.offset,
                   C.sizeof(S.QdsWindowConfig), S.QdsWindowConfig.scale.offset,
                   C.sizeof(S.QdsDecayConfig), S.QdsDecayConfig.scale.offset]


# -- refusals: every entry point checks before it launches anything
P = 1 << 20                                       # a pointer that nothing may follow


def view(p=P, strides=(8, 8, 8)):
    return S.QdsView(p, *strides)


def norm(**over):
    f = dict(abi_version=S.ABI_VERSION, dtype=S.BF16, weight_dtype=S.BF16, width=128, rows=4, eps=1e-6, group=0)
    f.update(over)
    return S.QdsNormConfig(*[f[n] for n, _ in S.QdsNormConfig._fields_])


def window(**over):
    f = dict(abi_version=S.ABI_VERSION, dtype=S.BF16, batch=2, length=100, heads=4, kv_heads=2, dim=64,
             window=10, sinks=1, scale=0.125)
    f.update(over)
    return S.QdsWindowConfig(*[f[n] for n, _ in S.QdsWindowConfig._fields_])


def decay(**over):
    f = dict(abi_version=S.ABI_VERSION, dtype=S.BF16, batch=2, length=100, heads=4, dim_k=64, dim_v=64, scale=0.125)
    f.update(over)
    return S.QdsDecayConfig(*[f[n] for n, _ in S.QdsDecayConfig._fields_])


def bytes_of(fn, cfg):
    n = C.c_uint64()
    return fn(C.byref(cfg), C.byref(n)), n.value


@pytest.mark.parametrize("over", [
    dict(abi_version=99), dict(dtype=3), dict(dtype=-1), dict(weight_dtype=S.F16), dict(width=0),
    dict(width=(1 << 20) + 1), dict(rows=-1), dict(rows=1 << 31), dict(eps=-1.0), dict(eps=float("nan")),
    dict(group=64), dict(group=128, width=192)])
def test_norm_refusals(lib, over):
    assert bytes_of(lib.qds_residual_norm_backward_workspace, norm(**over))[0] == S.ERR_INVALID_ARG
    assert lib.qds_residual_norm_fp8(C.byref(norm(**over)), P, 128, P, 128, P, P, P, P, None) == S.ERR_INVALID_ARG


def test_norm_refuses_pointers(lib):
    c = norm()
    assert lib.qds_residual_norm(None, P, 128, P, 128, P, P, P, P, None) == S.ERR_INVALID_ARG
    for missing in (1, 5, 6, 7, 8):
        a = [C.byref(c), P, 128, P, 128, P, P, P, P, None]
        a[missing] = None
        assert lib.qds_residual_norm(*a) == S.ERR_INVALID_ARG
        assert lib.qds_residual_norm_fp8(*a) == S.ERR_INVALID_ARG
    assert lib.qds_residual_norm(C.byref(norm(group=128)), P, 128, P, 128, P, P, P, P, None) == S.ERR_INVALID_ARG
    st, need = bytes_of(lib.qds_residual_norm_backward_workspace, c)
    assert st == S.OK and need > 0
    full = [C.byref(c), P, 128, P, 128, P, 128, P, P, P, P, P, need, None]
    short = list(full)
    short[12] = need - 1
    assert lib.qds_residual_norm_backward(*short) == S.ERR_WORKSPACE_TOO_SMALL
    for missing in (1, 5, 7, 8, 9, 10, 11):
        a = list(full)
        a[missing] = None
        assert lib.qds_residual_norm_backward(*a) == S.ERR_INVALID_ARG
    odd = list(full)
    odd[11] = P + 64                               # workspace: 256-byte aligned
    assert lib.qds_residual_norm_backward(*odd) == S.ERR_INVALID_ARG


WINDOW_BAD = [
    (dict(abi_version=0), S.ERR_INVALID_ARG), (dict(dtype=7), S.ERR_INVALID_ARG), (dict(dtype=S.F32), S.ERR_UNSUPPORTED),
    (dict(batch=-1), S.ERR_INVALID_ARG), (dict(length=-1), S.ERR_INVALID_ARG), (dict(heads=0), S.ERR_INVALID_ARG),
    (dict(kv_heads=0), S.ERR_INVALID_ARG), (dict(heads=5), S.ERR_INVALID_ARG), (dict(dim=0), S.ERR_INVALID_ARG),
    (dict(dim=12), S.ERR_UNSUPPORTED), (dict(dim=136), S.ERR_UNSUPPORTED), (dict(window=0), S.ERR_INVALID_ARG),
    (dict(sinks=-1), S.ERR_INVALID_ARG), (dict(window=1 << 30), S.ERR_INVALID_ARG),
    (dict(length=1 << 30), S.ERR_INVALID_ARG), (dict(scale=0.0), S.ERR_INVALID_ARG),
    (dict(scale=-1.0), S.ERR_INVALID_ARG), (dict(scale=float("nan")), S.ERR_INVALID_ARG),
    (dict(scale=float("inf")), S.ERR_INVALID_ARG), (dict(batch=1 << 24, heads=4), S.ERR_UNSUPPORTED)]


@pytest.mark.parametrize("over,status", WINDOW_BAD)
def test_window_refusals(lib, over, status):
    c = window(**over)
    assert bytes_of(lib.qds_window_backward_workspace, c)[0] == status
    assert bytes_of(lib.qds_window_step_workspace, c)[0] == status
    v = view()
    assert lib.qds_window_forward(C.byref(c), v, v, v, None, v, P, None) == status
    assert lib.qds_window_cache_fill(C.byref(c), v, v, None, P, P, None) == status


@pytest.mark.parametrize("bad", [view(None), view(P + 8), view(P, (4, 8, 8)), view(P, (8, 4, 8)), view(P, (8, 8, 4))])
def test_window_refuses_views(lib, bad):
    c, v = window(), view()
    for i in range(4):
        a = [v, v, v, v]
        a[i] = bad
        assert lib.qds_window_forward(C.byref(c), *a[:3], None, a[3], P, None) == S.ERR_INVALID_ARG
    st, need = bytes_of(lib.qds_window_backward_workspace, c)
    assert st == S.OK
    for i in range(8):
        a = [v] * 8
        a[i] = bad
        assert lib.qds_window_backward(C.byref(c), *a[:5], P, None, *a[5:], P, need, None) == S.ERR_INVALID_ARG
    assert lib.qds_window_backward(C.byref(c), *[v] * 5, P, None, *[v] * 3, P, need - 1, None) == S.ERR_WORKSPACE_TOO_SMALL
    assert lib.qds_window_backward(C.byref(c), *[v] * 5, None, None, *[v] * 3, P, need, None) == S.ERR_INVALID_ARG
    assert lib.qds_window_forward(C.byref(c), v, v, v, None, v, None, None) == S.ERR_INVALID_ARG


def test_window_step_refuses(lib):
    c, v = window(window=1 << 20), view()
    st, need = bytes_of(lib.qds_window_step_workspace, c)
    assert st == S.OK and need > 0
    ok = [C.byref(c), v, v, v, P, P, P, v, P, need, None]
    for i, bad in [(1, view(None)), (4, None), (5, P + 8), (6, None), (8, None), (8, P + 16)]:
        a = list(ok)
        a[i] = bad
        assert lib.qds_window_step(*a) == S.ERR_INVALID_ARG
    ok[9] = need - 1
    assert lib.qds_window_step(*ok) == S.ERR_WORKSPACE_TOO_SMALL


@pytest.mark.parametrize("over,status", [
    (dict(abi_version=0), S.ERR_INVALID_ARG), (dict(dtype=S.F32), S.ERR_UNSUPPORTED), (dict(dtype=9), S.ERR_INVALID_ARG),
    (dict(batch=-1), S.ERR_INVALID_ARG), (dict(length=-1), S.ERR_INVALID_ARG), (dict(heads=0), S.ERR_INVALID_ARG),
    (dict(dim_k=0), S.ERR_INVALID_ARG), (dict(dim_k=20), S.ERR_UNSUPPORTED), (dict(dim_v=136), S.ERR_UNSUPPORTED),
    (dict(scale=0.0), S.ERR_INVALID_ARG), (dict(scale=float("nan")), S.ERR_INVALID_ARG),
    (dict(batch=1 << 24, heads=2), S.ERR_UNSUPPORTED)])
def test_decay_refusals(lib, over, status):
    c, v = decay(**over), view()
    assert bytes_of(lib.qds_decay_forward_workspace, c)[0] == status
    assert bytes_of(lib.qds_decay_backward_workspace, c)[0] == status
    assert lib.qds_decay_forward(C.byref(c), v, v, v, P, None, None, v, P, P, 1 << 40, None) == status
    assert lib.qds_decay_step(C.byref(c), v, v, v, P, P, v, P, None) == status


def test_decay_refuses_pointers(lib):
    c, v = decay(batch=1, heads=1, length=5000), view()
    st, need = bytes_of(lib.qds_decay_forward_workspace, c)
    assert st == S.OK and need > 0
    ok = [C.byref(c), v, v, v, P, None, None, v, P, P, need, None]
    for i, bad in [(1, view(P + 2)), (2, view(None)), (3, view(P, (8, 1, 8))), (4, None), (7, view(None)), (9, None)]:
        a = list(ok)
        a[i] = bad
        assert lib.qds_decay_forward(*a) == S.ERR_INVALID_ARG
    ok[10] = need - 1
    assert lib.qds_decay_forward(*ok) == S.ERR_WORKSPACE_TOO_SMALL
    st, need = bytes_of(lib.qds_decay_backward_workspace, c)
    ok = [C.byref(c), v, v, v, v, P, None, None, None, v, v, v, None, P, need - 1, None]
    assert lib.qds_decay_backward(*ok) == S.ERR_WORKSPACE_TOO_SMALL
    ok[14] = need
    for i, bad in [(1, view(None)), (5, None), (9, view(P + 4)), (13, None)]:
        a = list(ok)
        a[i] = bad
        assert lib.qds_decay_backward(*a) == S.ERR_INVALID_ARG
    ok = [C.byref(c), v, v, v, P, P, v, P, None]
    for i, bad in [(1, view(P + 8)), (4, None), (5, None), (6, view(None)), (7, P + 4)]:
        a = list(ok)
        a[i] = bad
        assert lib.qds_decay_step(*a) == S.ERR_INVALID_ARG


def test_empty_calls_launch_nothing(lib):
    """No rows, no batch, no length: done without a GPU (and without pointers)."""
    none = view(None)
    assert lib.qds_residual_norm(C.byref(norm(rows=0)), None, 0, None, 0, None, None, None, None, None) == S.OK
    assert lib.qds_window_forward(C.byref(window(batch=0)), none, none, none, None, none, None, None) == S.OK
    assert lib.qds_window_forward(C.byref(window(length=0)), none, none, none, None, none, None, None) == S.OK
    assert lib.qds_window_step(C.byref(window(batch=0)), none, none, none, None, None, None, none, None, 0, None) == S.OK
    assert lib.qds_decay_step(C.byref(decay(batch=0)), none, none, none, None, None, none, None, None) == S.OK


def test_status_strings(lib):
    assert len({lib.qds_status_str(s) for s in (0, 1, 2, 4, 5)}) == 5
    assert lib.qds_status_str(77) == b"unknown status"


# -- the binding's own checks (they come before anything touches a GPU)
def test_binding_needs_a_gpu():
    x = torch.zeros(4, 128)
    with pytest.raises(RuntimeError, match="GPU"):
        S.residual_norm_forward(x, x, x[0])
    q = torch.zeros(1, 8, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(RuntimeError, match="GPU"):
        S.window_attention_forward(q, q, q, window=4)
    with pytest.raises(RuntimeError, match="GPU"):
        S.decay_attention_forward(q, q, q, torch.zeros(2))


def test_decay_has_no_gradient_of_its_decay():
    q = torch.zeros(1, 8, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="constant"):
        S.decay_attention(q, q, q, torch.zeros(2, requires_grad=True))


# -- index arithmetic
def slot_of(p, w, s):
    return p if p < s else s + (p - s) % w


@pytest.mark.parametrize("w,s", [(1, 0), (1, 3), (5, 0), (5, 2), (8, 8)])
def test_ring_holds_what_a_token_sees(w, s):
    """After the token at position p is written, the first min(p + 1, s + w)
    slots hold exactly the positions that it sees."""
    ring = {}
    for p in range(4 * (w + s) + 3):
        ring[slot_of(p, w, s)] = p
        seen = {j for j in range(p + 1) if p - j < w or j < s}
        assert {ring[i] for i in range(min(p + 1, w + s))} == seen


@pytest.mark.parametrize("w,s", [(1, 0), (5, 0), (5, 2), (8, 8)])
def test_ring_filled_from_a_prompt(w, s):
    """The fill kernel's rule for a slot gives the latest position below n that belongs in it."""
    for n in range(0, 4 * (w + s) + 2):
        want = {}
        for p in range(n):
            want[slot_of(p, w, s)] = p
        got, last = {}, n - 1
        for slot in range(w + s):
            if last >= slot:
                got[slot] = slot if slot < s else last - (last - slot) % w
        assert got == want
