"""The selective block's operators on the CPU: the limits of launches and sizes, and what the binding
does before any GPU work."""
import ctypes as C
import os

import pytest

torch = pytest.importorskip("torch")

from paper_2202_01258_amd import seq as S  # noqa: E402
from test_seq_block_abi import P, bytes_of, rows, scan  # noqa: E402


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
