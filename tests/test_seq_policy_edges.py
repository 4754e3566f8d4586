"""The sequence policy's rollouts at the edges: prompts whose lengths pass the tokens given."""
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu


def test_prompt_lengths_beyond_the_tokens():
    """Lengths are clamped to the tokens there are, for the caches, the states and the positions alike."""
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2202_01258_amd import seq_policy as P
    torch.manual_seed(0)
    policy = P.SequencePolicy(window=5)
    tokens = torch.randn(3, 13, policy.width, device="cuda").to(torch.bfloat16)
    as_int = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    want, got = P.Rollout(policy, 3), P.Rollout(policy, 3)
    want.prompt(tokens[:, :10], as_int(10, 0, 4))
    got.prompt(tokens[:, :10], as_int(25, -3, 4))
    assert torch.equal(got.pos, want.pos) and want.pos.tolist() == [10, 0, 4]
    for t in range(10, 13):
        assert torch.equal(got.step(tokens[:, t]), want.step(tokens[:, t]))


def test_a_rollout_keeps_its_weights():
    """A rollout acts with the policy as it was when the rollout began: fitting goes on beside it."""
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2202_01258_amd import seq_policy as P
    torch.manual_seed(0)
    policy = P.SequencePolicy(window=5)
    tokens = torch.randn(3, 4, policy.width, device="cuda").to(torch.bfloat16)
    want, got = P.Rollout(policy, 3), P.Rollout(policy, 3)
    expected = [want.step(tokens[:, t]) for t in range(4)]
    with torch.no_grad():
        for p in policy.parameters():
            p.mul_(1.5)
    for t in range(4):
        assert torch.equal(got.step(tokens[:, t]), expected[t])
