"""The token policy's funnel where a member cannot draw, or a reward is no number: the run says so."""
import math

import pytest
import torch

from test_gpu_rollout_loop import CFG, DEV

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def weights():
    from paper_2512_15347_amd import rollout
    return rollout.make_weights(CFG, seed=9)


def test_nothing_to_draw_from_is_an_error(lib, weights):
    from paper_2512_15347_amd import rollout
    print("a mask that allows nothing", flush=True)
    allow = torch.zeros(1, -(-CFG["vocab"] // 32), dtype=torch.int32, device=DEV)
    decoder = rollout.Decoder(CFG, weights, rows=4)
    with pytest.raises(lib.PgError) as e:
        rollout.sample_groups(decoder, [[5, 6]], 4, 3, [(1, 2)], 1, torch.ones(CFG["vocab"], device=DEV), allow=allow)
    assert e.value.status == lib.PG_EINVAL


def test_logits_of_nan_are_an_error(lib, weights):
    from paper_2512_15347_amd import rollout
    print("logits of NaN", flush=True)
    head = weights["head"].clone()
    head[7] = math.nan
    decoder = rollout.Decoder(CFG, dict(weights, head=head), rows=4)
    with pytest.raises(lib.PgError) as e:
        rollout.sample_groups(decoder, [[5, 6]], 4, 3, [], 1, torch.ones(CFG["vocab"], device=DEV))
    assert e.value.status == lib.PG_EINVAL


def test_a_reward_of_nan_at_a_checkpoint_is_an_error(lib, weights):
    from paper_2512_15347_amd import rollout
    print("rewards of NaN", flush=True)
    for schedule in ([(0, 3), (2, 2)], [(2, 2)]):           # the first of two checkpoints, or the only one
        decoder = rollout.Decoder(CFG, weights, rows=8)
        with pytest.raises(lib.PgError) as e:
            rollout.sample_groups(decoder, [[5, 6], [9]], 4, 4, schedule, 1, torch.full((CFG["vocab"],), math.nan, device=DEV))
        assert e.value.status == lib.PG_ENAN
