"""The sequence policy fitted to an archive's elites: operators together."""
import pytest

torch = pytest.importorskip("torch")

from paper_2202_01258_amd import workloads as W  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def setup():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2202_01258_amd import qd, seq_policy as P
    torch.manual_seed(0)
    archive = qd.Archive(W.workload("mlp64_cvt_b8192", batch=512, T=40, C=10000, iso_sigma=0.1, line_sigma=0.5))
    archive.generations(1, 60)
    env = P.environment(archive)
    geno, desc = P.elites(archive)
    states, actions = P.episodes(geno, 64, env, 40)
    return P, env, desc, states, actions


def test_episodes_are_the_elites_own(setup):
    """The elites' descriptors from the torch rollout: the library's, up to fp32 order."""
    P, env, desc, states, actions = setup
    a_mat, b_mat, _ = env
    last = torch.tanh(states[:, -1] @ a_mat.T + actions[:, -1] @ b_mat.T)
    got = P.descriptors(torch.cat([states[:, 1:], last[:, None]], 1))
    assert desc.shape[0] > 10 and (got - desc).abs().max() < 1e-4


def test_fit_lowers_the_loss(setup):
    P, _, desc, states, actions = setup
    torch.manual_seed(1)
    losses = P.fit(P.SequencePolicy(window=16), desc, states, actions, iterations=80, batch=32)
    assert losses.isfinite().all()
    assert losses[-5:].mean() < 0.5 * losses[:5].mean()


def test_steps_and_prompts_follow_the_whole_sequence(setup):
    """Token by token, and from a prompt of mixed lengths on: the actions of one
    forward call, up to the roundings of bfloat16 layers (actions are in [-1, 1])."""
    P, _, desc, states, _ = setup
    torch.manual_seed(2)
    policy = P.SequencePolicy(window=9)
    tokens = policy.tokens(desc[:6], states[:6]).detach()
    with torch.no_grad():
        want = policy(tokens)
    run = P.Rollout(policy, 6)
    got = torch.stack([run.step(tokens[:, t]) for t in range(tokens.shape[1])], 1)
    assert (got - want).abs().max() < 0.05 and (got - want).abs().mean() < 0.005
    lengths = torch.tensor([1, 5, 9, 10, 11, 30], dtype=torch.int32, device="cuda")
    run = P.Rollout(policy, 6)
    run.prompt(tokens[:, :30], lengths)
    rows = torch.arange(6, device="cuda")
    for step in range(5):
        at = lengths.long() + step
        got = run.step(tokens[rows, at])
        assert (got - want[rows, at]).abs().max() < 0.05


def test_eight_bits_stay_near(setup):
    P, _, desc, states, _ = setup
    torch.manual_seed(3)
    policy = P.SequencePolicy(window=9)
    tokens = policy.tokens(desc[:6], states[:6]).detach()
    plain, low = P.Rollout(policy, 6), P.Rollout(policy, 6)
    for t in range(12):
        a, b = plain.step(tokens[:, t]), low.step(tokens[:, t], eight_bits=True)
        # e4m3 keeps 4 bits: each projection is off by some percent, in random directions
        assert (a - b).abs().mean() < 0.05


def test_a_rollout_step_in_a_graph(setup):
    """One captured step, replayed along an episode, gives the eager actions."""
    P, _, desc, states, _ = setup
    torch.manual_seed(4)
    policy = P.SequencePolicy(window=9)
    tokens = policy.tokens(desc[:6], states[:6]).detach()
    eager = P.Rollout(policy, 6)
    want = [eager.step(tokens[:, t]) for t in range(15)]
    run = P.Rollout(policy, 6)
    token = tokens[:, 0].clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        P.Rollout(policy, 6).step(token)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = run.step(token)
    run.pos.zero_()
    for s in run.state:
        s.zero_()
    for t in range(15):
        token.copy_(tokens[:, t])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, want[t]), t
