"""Workspaces asked for once, for the largest call of a rollout, and used by all of its calls."""
import pytest
import torch

from test_gpu_rollout import DEV, dev, say

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("vocab", [17, 4097, 65537])
@pytest.mark.parametrize("most", [60, 700, 1300])
def test_draws_stay_inside_the_scratch_of_the_largest_call(lib, most, vocab):
    say(f"scratch of {most} rows of {vocab} tokens")
    x = torch.randn(most, vocab, device=DEV, generator=torch.Generator(device=DEV).manual_seed(most))
    size = lib.pg_sample_scratch_floats(most, vocab)
    guard = torch.full((size + 4096,), 12345.0, device=DEV)
    token, logp = torch.empty(most, dtype=torch.int32, device=DEV), torch.empty(most, device=DEV)
    first = None
    for rows in (most, 1281, 1280, 700, 640, 641, 427, 320, 48, 5, 1):
        if rows > most:
            continue
        lib.pg_sample_tokens(lib.Logits(x[:rows]), None, 9, 1, None, token[:rows], logp[:rows], guard[:size])
        assert (guard[size:] == 12345.0).all(), rows
        first = token.clone() if first is None else first
        assert torch.equal(token[:rows], first[:rows])
