"""The sequence policy's arguments with selective layers, norms behind branches and dropout (CPU)."""
import pytest

torch = pytest.importorskip("torch")

from paper_2202_01258_amd import seq as S  # noqa: E402
from paper_2202_01258_amd import seq_policy as P  # noqa: E402


@pytest.mark.parametrize("p", [1.0, -0.1, 1.5, 1 - 2.0 ** -18, float("nan"), float("inf")])
def test_policy_refuses_a_dropout_that_its_layers_refuse(p):
    with pytest.raises(ValueError, match="probability"):
        P.SequencePolicy(device="cpu", dropout=p)


@pytest.mark.parametrize("p", [0.0, 0.1, 1 - 2.0 ** -16])
def test_policy_takes_a_dropout(p):
    policy = P.SequencePolicy(device="cpu", mixers=("scan",), blocks=1, dropout=p, seed=7)
    assert policy.dropout == p and ("rng" in dict(policy.named_buffers())) == (p > 0)
    assert S.dropout_rng(7, 0, "cpu").tolist() == [7, 0]


@pytest.mark.parametrize("scale", [float("nan"), float("inf")])
def test_policy_refuses_a_scale_that_is_not_finite(scale):
    with pytest.raises(ValueError, match="residual_scale"):
        P.SequencePolicy(device="cpu", post_norm=True, residual_scale=scale)
