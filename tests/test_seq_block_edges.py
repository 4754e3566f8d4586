"""The selective block's operators on the CPU: the limits of launches and sizes, and what the binding
does before any GPU work."""
import ctypes as C
import os

import pytest

torch = pytest.importorskip("torch")
import torch.autograd.forward_ad as forward_ad  # noqa: E402

from paper_2202_01258_amd import seq as S  # noqa: E402
from test_seq_block_abi import P, bytes_of, conv, rows, scan  # noqa: E402


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(S.LIB_PATH):
        pytest.skip("libqdseq.so not built")
    return S.lib()


# 64 columns for each workgroup of 256 threads, and 2^24 - 1 workgroups: 2^30 - 64 columns.  These would
# take one workgroup more, 2^32 threads, of which HIP leaves some out without an error.
@pytest.mark.parametrize("batch,width", [(34636831, 31), (282638, 3799), (32767, 32769)])
def test_scan_step_refuses_a_launch_of_2_to_the_32_threads(lib, batch, width):
    columns = batch * width
    assert (1 << 30) - 63 <= columns < 1 << 30 and -(-columns // 64) == 1 << 24
    c, r = scan(batch=batch, width=width, length=0), rows()
    assert lib.qds_selective_scan_step(C.byref(c), r, r, P, r, r, P, r, P, P, P, P, None) == S.ERR_UNSUPPORTED


# A workgroup has 64 columns of one batch element: 2^24 - 1 of them are what a launch takes.  Many columns
# are not cut into pieces, so nothing else limits them.
@pytest.mark.parametrize("batch,length,width,status", [
    (8192, 8, 1023, S.OK), (8192, 8, 1024, S.OK), (16384, 1, 512, S.OK), (16384, 100, 2048, S.OK), (1 << 23, 2, 1, S.OK),
    ((1 << 24) - 1, 1, 64, S.OK), (1 << 24, 1, 1, S.ERR_UNSUPPORTED), (1 << 23, 1, 65, S.ERR_UNSUPPORTED)])
@pytest.mark.parametrize("states", [1, 16, 32])
def test_scan_takes_many_columns(lib, batch, length, width, status, states):
    c = scan(batch=batch, length=length, width=width, states=states)
    assert bytes_of(lib.qds_selective_scan_workspace, c)[0] == status
    assert bytes_of(lib.qds_selective_scan_backward_workspace, c)[0] == status


# -- what the binding does without a GPU: the plain calls are stood in for
@pytest.fixture
def stand_ins(monkeypatch):
    """The plain forward calls, giving new tensors of the right shapes as the library does; what
    selective_scan_forward was asked to keep is returned."""
    kept = []

    def scan_forward(u, delta, a, b, c, skip=None, gate=None, bias=None, state=None, lengths=None, keep=False):
        kept.append(keep)
        return u.new_zeros(u.shape), u.new_zeros(u.shape[0], *a.shape), u.new_zeros(8) if keep else None

    monkeypatch.setattr(S, "selective_scan_forward", scan_forward)
    monkeypatch.setattr(S, "causal_conv_forward", lambda x, w, *_: (x.new_zeros(x.shape), x.new_zeros(x.shape[0], 3, x.shape[2])))
    monkeypatch.setattr(S, "branch_norm_forward", lambda x, *_: (x.new_zeros(x.shape), x.new_zeros(x.shape), x.new_zeros(2, *x.shape[:-1])))
    monkeypatch.setattr(S, "dropout_forward", lambda x, *_: x.new_zeros(x.shape))
    return kept


X, W, A, N = torch.ones(2, 5, 8), torch.ones(4, 8), torch.ones(8, 4), torch.ones(2, 5, 4)
NAMES = ("u", "delta", "a", "b", "c")
RNG = torch.zeros(2, dtype=torch.int64)


@pytest.mark.parametrize("call", [lambda x: S.causal_conv(x, W), lambda x: S.selective_scan(x, X, A, N, N),
                                  lambda x: S.selective_scan(X, X, A, N, N, gate=x), lambda x: S.branch_norm(x, None, X, W[0], W[0]),
                                  lambda x: S.dropout(x, RNG, 0.5)])
@pytest.mark.parametrize("mode", [torch.enable_grad, torch.no_grad])
def test_forward_mode_is_refused(stand_ins, call, mode):
    """There is no forward-mode derivative; torch.no_grad does not switch forward mode off, so a tangent
    must not get lost there either."""
    with forward_ad.dual_level(), mode():
        with pytest.raises(NotImplementedError, match="jvp"):
            call(forward_ad.make_dual(X, torch.ones_like(X)))


def test_scan_keeps_nothing_without_gradients(stand_ins):
    with torch.no_grad():
        S.selective_scan(X.clone().requires_grad_(), X, A, N, N)
    S.selective_scan(X.clone().requires_grad_(), X, A, N, N)
    assert stand_ins == [False, True]


@pytest.mark.parametrize("which", ["u", "delta", "a", "b", "c", "skip", "gate", "bias", "state"])
def test_scan_keeps_only_for_inputs_with_gradients(stand_ins, which):
    """Frozen layers and evaluations with gradients on have no backward pass either."""
    tensors = dict(u=X, delta=X, a=A, b=N, c=N, skip=W[0], gate=X, bias=W[0], state=torch.ones(2, 8, 4))
    assert not S.selective_scan(**tensors, lengths=torch.ones(2, dtype=torch.int32))[0].requires_grad
    tensors[which] = tensors[which].clone().requires_grad_()
    assert S.selective_scan(**tensors)[0].requires_grad
    assert S.selective_scan(**{k: v if k == which or k in NAMES else None for k, v in tensors.items()})[0].requires_grad
    assert stand_ins == [False, True, True]


def test_scan_scratch_memory(lib):
    """Shares of db and dc, 2 * 16 floats for 64 columns of a row, are nearly all of it; of da, dskip and dbias there
    is one for each of the 32 episodes, which are whole.  Counts that leave places in four lanes add what the threads
    of 32 * 16 workgroups may save: 2 * 4 + 2 floats each."""
    shares, rest = 32 * 1000 * 16 * 2 * 16 * 4, 32 * 1024 * (16 + 2) * 4
    assert bytes_of(lib.qds_selective_scan_backward_workspace, scan(batch=32, length=1000, width=1024))[1] == shares + rest
    saved = 32 * 16 * 256 * 10 * 4
    assert bytes_of(lib.qds_selective_scan_backward_workspace,
                    scan(batch=32, length=1000, width=1024, states=13))[1] == shares + rest + saved


@pytest.mark.parametrize("batch,length,status", [(1, 1 << 25, S.OK), (1 << 12, 1 << 13, S.OK), (3, 11184810, S.OK),
                                                 (1, (1 << 25) + 1, S.ERR_UNSUPPORTED), (1 << 13, (1 << 12) + 1, S.ERR_UNSUPPORTED)])
@pytest.mark.parametrize("states", [1, 16, 32])
def test_scan_backward_takes_2_to_the_25_rows(lib, batch, length, status, states):
    """batch times length as the header has it; the forward pass takes more."""
    c = scan(batch=batch, length=length, states=states)
    assert bytes_of(lib.qds_selective_scan_backward_workspace, c)[0] == status
    assert bytes_of(lib.qds_selective_scan_workspace, c)[0] == S.OK


def test_backward_passes_refuse_gradients_in_place(lib):
    """A gradient is written where other workgroups (the convolution's next rows) or a later look (the scan's
    blocks that are gone through again) still read the inputs.  With no address that could be followed the call ends
    at the check, or at the launch for want of a device."""
    c = conv()
    need = bytes_of(lib.qds_causal_conv_backward_workspace, c)[1]
    for dy, x in ((2 * P, P), (P, 2 * P)):            # dx is at P
        assert lib.qds_causal_conv_backward(C.byref(c), rows(dy), rows(x), P, P, P, P, None, rows(), P, P, P + 4096, P, need,
                                            None) == S.ERR_INVALID_ARG
    c = scan()
    need = bytes_of(lib.qds_selective_scan_backward_workspace, c)[1]
    for out in range(3):                              # du, ddelta, dgate
        for place in range(4):                        # dout, u, delta, gate
            do, u, delta, gate = [rows((16 + i) * P) for i in range(4)]
            to = [(32 + i) * P for i in range(3)]
            to[out] = (16 + place) * P
            assert lib.qds_selective_scan_backward(
                C.byref(c), do, u, delta, P, rows(), rows(), P, gate, P, P, P, None, to[0], to[1], 40 * P, 41 * P, 42 * P, 43 * P,
                to[2], 44 * P, 45 * P, 46 * P, need, None) == S.ERR_INVALID_ARG
