"""The selective block's operators on the CPU: the limits of launches and sizes, and what the binding
does before any GPU work."""
import ctypes as C
import os

import pytest

torch = pytest.importorskip("torch")

from paper_2202_01258_amd import seq as S  # noqa: E402
from test_seq_block_abi import P, rows, scan  # noqa: E402


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
