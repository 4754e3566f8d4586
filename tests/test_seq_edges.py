"""libqdseq.so on the CPU: empty calls, the sizes that it accepts, and the
scratch memory and work items that it plans."""
import ctypes as C
import os
import random
import shutil
import subprocess
import sys

import pytest

from paper_2202_01258_amd import seq as S

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 1 << 20                                       # a pointer that nothing may follow


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(S.LIB_PATH):
        pytest.skip("libqdseq.so not built")
    return S.lib()


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


# -- no rows, no batch: every query answers, and a call without outputs launches nothing.
# In a process of its own, as a fault here would end the test runner.
EMPTY = """
import sys
sys.path[:0] = [{root!r}, {tests!r}]
import ctypes as C
from paper_2202_01258_amd import seq as S
import test_seq_edges as T
lib, none = S.lib(), T.view(None)
for over in (dict(length=0), dict(batch=0), dict(length=0, sinks=0), dict(length=0, window=1 << 20, sinks=1 << 20)):
    st, need = T.bytes_of(lib.qds_window_backward_workspace, T.window(**over))
    assert (st, need) == (S.OK, 0), (over, st, need)
    assert T.bytes_of(lib.qds_window_step_workspace, T.window(**over))[0] == S.OK
    c = T.window(**over)
    assert lib.qds_window_forward(C.byref(c), none, none, none, None, none, None, None) == S.OK
    assert lib.qds_window_backward(C.byref(c), *[none] * 5, None, None, *[none] * 3, None, 0, None) == S.OK
    assert lib.qds_window_cache_fill(C.byref(c), none, none, None, None, None, None) == S.OK
for over in (dict(length=0), dict(batch=0)):
    for query in (lib.qds_decay_forward_workspace, lib.qds_decay_backward_workspace):
        assert T.bytes_of(query, T.decay(**over)) == (S.OK, 0)
c = T.decay(batch=0)
assert lib.qds_decay_forward(C.byref(c), none, none, none, None, None, None, none, None, None, 0, None) == S.OK
assert lib.qds_decay_backward(C.byref(c), *[none] * 4, None, None, None, None, *[none] * 3, None, None, 0, None) == S.OK
assert T.bytes_of(lib.qds_residual_norm_backward_workspace, T.norm(rows=0))[0] == S.OK
print("all answered")
"""


def test_empty_calls(lib):
    done = subprocess.run([sys.executable, "-c", EMPTY.format(root=ROOT, tests=os.path.join(ROOT, "tests"))],
                          capture_output=True, text=True)
    assert done.returncode == 0 and "all answered" in done.stdout, (done.returncode, done.stderr)


# -- a launch has fewer than 2^32 threads in a dimension; HIP takes more without an error
# and leaves workgroups out, so that outputs would stay unwritten
def window_calls(lib, c):
    v = view()
    return {"forward": lib.qds_window_forward(C.byref(c), v, v, v, None, v, P, None),
            "backward": lib.qds_window_backward(C.byref(c), *[v] * 5, P, None, *[v] * 3, P, 1 << 62, None),
            "query": bytes_of(lib.qds_window_backward_workspace, c)[0]}


@pytest.mark.parametrize("over", [
    dict(batch=16, heads=4, kv_heads=1, length=1 << 25), dict(batch=1 << 12, heads=1, kv_heads=1, length=1 << 19),
    dict(batch=1 << 24, heads=1, kv_heads=1, length=1), dict(batch=1 << 11, heads=2, kv_heads=1, length=1 << 19, dim=128)])
def test_window_refuses_more_work_than_a_launch_takes(lib, over):
    assert set(window_calls(lib, window(**over)).values()) == {S.ERR_UNSUPPORTED}


@pytest.mark.parametrize("over", [
    dict(batch=16, heads=4, kv_heads=1, length=(1 << 25) - 32), dict(batch=(1 << 12) - 1, heads=1, kv_heads=1, length=1 << 19, sinks=0),
    dict(batch=(1 << 24) - 1, heads=1, kv_heads=1, length=1, sinks=0)])
def test_window_takes_what_a_launch_takes(lib, over):
    assert bytes_of(lib.qds_window_backward_workspace, window(**over))[0] == S.OK


def test_steps_have_no_length(lib):
    """The step does not use `length`, so nothing is refused for it."""
    assert bytes_of(lib.qds_window_step_workspace, window(batch=64, length=(1 << 30) - 1))[0] == S.OK
    for batch, status in (((1 << 24) - 1, S.OK), (1 << 24, S.ERR_UNSUPPORTED)):
        assert bytes_of(lib.qds_window_step_workspace, window(batch=batch, heads=1, kv_heads=1))[0] == status


def test_decay_refuses_more_work_than_a_launch_takes(lib):
    for batch, status in (((1 << 24) - 1, S.OK), (1 << 24, S.ERR_UNSUPPORTED)):
        c, v = decay(batch=batch, heads=1), view()
        assert bytes_of(lib.qds_decay_forward_workspace, c)[0] == status
        assert bytes_of(lib.qds_decay_backward_workspace, c)[0] == status
        if status != S.OK:
            assert lib.qds_decay_forward(C.byref(c), v, v, v, P, None, None, v, P, P, 1 << 40, None) == status
            assert lib.qds_decay_step(C.byref(c), v, v, v, P, P, v, P, None) == status


# -- the backward pass over keys: its work items, and the sums that cut blocks leave
@pytest.fixture(scope="module")
def replay(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("g++ not available")
    exe = tmp_path_factory.mktemp("plan") / "replay"
    src = os.path.join(ROOT, "tests", "helpers", "seq_plan_replay.cpp")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", src, "-o", str(exe)], check=True)

    def run(configs):
        """(items, sums, first_cut, band_cut) of each (batch, length, heads, kv_heads, dim, window, sinks)."""
        out = subprocess.run([str(exe)] + [str(x) for c in configs for x in c], capture_output=True, text=True)
        assert out.returncode == 0, out.stdout[-400:]
        return [tuple(map(int, line.split())) for line in out.stdout.splitlines()]

    return run


LENGTHS = [0, 1, 31, 64, 127, 128, 129, 300, 1000, 4096, 5001]


@pytest.mark.parametrize("window", [1, 33, 250, 1024, 1 << 20])
@pytest.mark.parametrize("sinks", [0, 1, 128, 129, 700, 1 << 20])
def test_work_items_cover_everything_once(replay, window, sinks):
    replay([(b, t, heads, kv, 64, window, sinks) for t in LENGTHS
            for b, heads, kv in ((0, 1, 1), (1, 1, 1), (2, 8, 2), (3, 6, 1), (64, 16, 16), (600, 4, 4))])


def backward_bytes(lib, c):
    """Scratch memory beside a float per row and query head."""
    st, need = bytes_of(lib.qds_window_backward_workspace, c)
    assert st == S.OK
    delta = c.batch * c.heads * c.length * 4
    return need - (delta + 255) // 256 * 256


def of(c):
    return (c.batch, c.length, c.heads, c.kv_heads, c.dim, c.window, c.sinks)


def test_scratch_memory_is_for_cut_blocks_only(lib, replay):
    """Blocks that are not cut write their gradients themselves."""
    wide = dict(batch=2, length=8192, heads=16, kv_heads=16, dim=128, window=1024)
    assert backward_bytes(lib, window(**wide, sinks=0)) == 0
    assert backward_bytes(lib, window(batch=64, length=16384, heads=8, kv_heads=8, dim=128, window=1024, sinks=0)) == 0
    configs = [window(**wide, sinks=16), window(**wide, sinks=0), window(batch=1, length=3000, window=64, sinks=0),
               window(batch=1, length=3000, window=64, sinks=300), window(batch=1, length=20000, window=2000, sinks=1)]
    for c, (items, sums, first_cut, band_cut) in zip(configs, replay([of(c) for c in configs])):
        columns = 64 if c.dim <= 64 else 128
        want = c.batch * c.kv_heads * sums * 2 * 128 * columns * 4
        assert backward_bytes(lib, c) == (want + 255) // 256 * 256
        if c.sinks == 0:
            assert first_cut == 1


@pytest.mark.parametrize("shape", [
    dict(batch=64, length=4096, heads=16, kv_heads=16, dim=128, window=256, sinks=1),
    dict(batch=256, length=1000, heads=8, kv_heads=8, dim=64, window=64, sinks=1),
    dict(batch=64, length=4096, heads=8, kv_heads=8, dim=64, window=16, sinks=4096)])
def test_first_blocks_stay_whole_where_lists_fill_the_card(lib, shape):
    assert backward_bytes(lib, window(**shape)) == 0


def test_scratch_memory_does_not_grow_with_the_lists(replay):
    """Pieces that leave sums: at most ten for each of the 512 places of the card.  (A first block's pieces
    are a quarter of a place's share of the work or more, rounded down to no less than a fifth; a block is
    cut into less than twice as many as that gives.)"""
    rng = random.Random(5)
    size = lambda most: int(2 ** rng.uniform(0, most))  # noqa: E731
    configs = []
    for _ in range(1500):
        kv, group = rng.choice([1, 1, 2, 4, 8, 16]), rng.choice([1, 1, 2, 3, 8])
        configs.append((size(10), size(13), kv * group, kv, 64, size(14), rng.choice([0, 1, size(14)])))
    for i in range(0, len(configs), 300):
        for c, (_, sums, _, _) in zip(configs[i:], replay(configs[i:i + 300])):
            assert c[0] * c[3] * sums <= 10 * 512, c


# -- rows far apart (the binding copies such tensors)
def test_rows_too_far_apart_are_refused(lib):
    v, far = view(), view(P, (8, 1 << 23, 8))
    c = window()
    for i in (1, 2):
        a = [v, v, v]
        a[i] = far
        assert lib.qds_window_forward(C.byref(c), *a, None, v, P, None) == S.ERR_UNSUPPORTED
    for i in range(4):
        a = [v] * 5
        a[i] = far
        assert lib.qds_window_backward(C.byref(c), *a, P, None, *[v] * 3, P, 1 << 40, None) == S.ERR_UNSUPPORTED
    c = decay()
    for i in range(3):
        a = [v] * 3
        a[i] = far
        assert lib.qds_decay_forward(C.byref(c), *a, P, None, None, v, P, P, 1 << 40, None) == S.ERR_UNSUPPORTED
    # a single row's stride means nothing: such a call is refused for other reasons only
    c = decay(length=1)
    assert lib.qds_decay_forward(C.byref(c), far, far, far, P, None, None, view(None), P, P, 1 << 40, None) == S.ERR_INVALID_ARG
