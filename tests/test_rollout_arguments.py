"""CPU-only: what the token policy's funnel refuses before it touches the device."""
import types

import pytest
import torch

from paper_2512_15347_amd import rollout

DECODER = types.SimpleNamespace(cfg=dict(max_len=64, vocab=50))      # refused calls need no more of it


def call(prompts, members, steps, schedule):
    return rollout.sample_groups(DECODER, prompts, members, steps, schedule, 1, torch.ones(50))


@pytest.mark.parametrize("schedule", [[(15, 8), (3, 5)], [(3, 8), (3, 5)], [(3, 5), (9, 6)], [(9, 6), (3, 5)], [(3, 13)], [(3, 0)]])
def test_schedules_that_are_no_funnel(schedule):
    """12 members, 20 steps: counts have to fall in the order of the steps, one count a step."""
    with pytest.raises(ValueError):
        call([[1, 2]], 12, 20, schedule)


@pytest.mark.parametrize("schedule", [[(3, 8), (15, 5)], [(15, 5), (3, 8)], [(19, 12)], [(3, 8), (25, 5)], []])
def test_schedules_in_any_order(schedule):
    with pytest.raises(AttributeError):                                # accepted: the next thing asked for is the decoder's cache
        call([[1, 2]], 12, 20, schedule)


def test_tokens_and_rewards_that_do_not_fit_the_vocabulary():
    for prompts in ([[1, 2], [3, 50]], [[-1]]):
        with pytest.raises(ValueError):
            call(prompts, 4, 3, [])
    for reward in (torch.ones(49), torch.ones(51), torch.ones(50, 1)):
        with pytest.raises(ValueError):
            rollout.sample_groups(DECODER, [[1]], 4, 3, [], 1, reward)
