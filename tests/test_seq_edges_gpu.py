"""The sequence operators on the GPU at the edges of what they accept: no rows,
values far from 1, very many rows, rows far apart.

Tolerances as in test_seq_gpu.py: bounds worked out element by element from
the kernels' roundings, against definitions in 64 bits.
"""
import math

import pytest

torch = pytest.importorskip("torch")

from paper_2202_01258_amd import seq as S  # noqa: E402
from test_seq_gpu import BF16, F16, F32, SINGLE, TINY, U, decay_exact, norm_exact, qkv, rand, within  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


# ---------------------------------------------------------------------------
# No rows, no batch
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("b,t", [(2, 0), (0, 7), (0, 0)])
def test_training_on_nothing(b, t):
    """Empty tensors through autograd: empty gradients, and the given gradient of a state."""
    q, k, v = (torch.empty(b, t, h, 64, dtype=BF16, device="cuda", requires_grad=True) for h in (4, 2, 2))
    S.window_attention(q, k, v, 10, 1).sum().backward()
    assert [x.grad.shape for x in (q, k, v)] == [x.shape for x in (q, k, v)]
    q, k, v = (torch.empty(b, t, 2, 64, dtype=BF16, device="cuda", requires_grad=True) for _ in range(3))
    state = rand(b, 2, 64, 64, seed=1).requires_grad_()
    o, last = S.decay_attention(q, k, v, torch.full((2,), -0.1, device="cuda"), state)
    (o.float().sum() + (last * 2).sum()).backward()
    assert (state.grad == 2).all() and q.grad.shape == q.shape
    x = torch.empty(b, t, 64, device="cuda", requires_grad=True)
    w = torch.ones(64, device="cuda", requires_grad=True)
    y, h = S.residual_norm(x, None, w)
    (y.sum() + h.sum()).backward()
    assert x.grad.shape == x.shape and (w.grad == 0).all()
