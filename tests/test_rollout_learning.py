"""What the rollouts of a token policy may be learnt from: refusals on the host, before anything is run."""
import pytest

from paper_2512_15347_amd import rollout


@pytest.mark.parametrize("call", [rollout.token_logprobs, rollout.policy_gradient])
@pytest.mark.parametrize("penalties", [(1.1, 0.0, 0.0), (1.0, 0.1, 0.0), [1, 0, -0.5]])
def test_rollouts_drawn_with_penalties_are_refused(call, penalties):
    """Their log-probs are those of adjusted logits: a ratio to the decoder's own would be another policy's."""
    with pytest.raises(ValueError, match="penalties"):
        call(None, dict(penalties=penalties))


def test_penalties_that_change_nothing_are_none():
    for penalties in (None, (1.0, 0.0, 0.0), [1, 0, 0]):
        rollout._without_penalties(dict(penalties=penalties))
    rollout._without_penalties({})
