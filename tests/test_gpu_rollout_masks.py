"""Mask indices that no mask has, and outputs beside the logits."""
import math

import pytest
import torch

from test_gpu_rollout import DEV, dev, say

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocab", [1, 40, 2049, 9001])
def test_an_index_that_no_mask_has_allows_nothing(lib, vocab, dtype):
    say(f"masks out of range, {vocab} tokens")
    rows = [0, -1, 2, -2, 1, 2 ** 31 - 1, -2 ** 31]          # two masks; -1: no mask
    n = len(rows)
    x = torch.randn(n, vocab, device=DEV, generator=torch.Generator(device=DEV).manual_seed(vocab)).to(dtype)
    allow = torch.full((2, (vocab + 31) // 32), -1, dtype=torch.int32, device=DEV)
    d = lib.Logits(x, allow=allow, allow_row=dev(rows))
    out = torch.zeros(n, vocab, device=DEV)
    lib.pg_logits_adjust(d, out)
    token, logp = torch.full((n,), -7, dtype=torch.int32, device=DEV), torch.zeros(n, device=DEV)
    scratch = torch.empty(d.scratch, device=DEV)
    for t in (None, torch.zeros(n, device=DEV)):
        lib.pg_sample_tokens(d, t, 3, 4, None, token, logp, scratch)
        for r, m in enumerate(rows):
            if m in (-1, 0, 1):
                assert torch.equal(out[r], x[r].float()) and 0 <= int(token[r]) < vocab and math.isfinite(float(logp[r]))
            else:
                assert (out[r] == -math.inf).all() and int(token[r]) == -1 and float(logp[r]) == -math.inf


def test_rows_between_the_logits_rows_may_be_written(lib):
    """Columns of one allocation, above and below, and blocks side by side."""
    say("adjusting into the other half of the rows")
    g = torch.Generator(device=DEV).manual_seed(3)
    wide = torch.randn(5, 2 * 3001, device=DEV, generator=g)
    keep = wide.clone()
    for lo, to in ((0, 3001), (3001, 0)):
        x, out = wide[:, lo:lo + 3001], wide[:, to:to + 3001]
        lib.pg_logits_adjust(lib.Logits(x), out)
        assert torch.equal(out, x) and torch.equal(x, keep[:, :3001])
    two = torch.randn(10, 3001, device=DEV, generator=g)
    keep = two.clone()
    lib.pg_logits_adjust(lib.Logits(two[5:]), two[:5])
    assert torch.equal(two[:5], keep[5:]) and torch.equal(two[5:], keep[5:])
    lib.pg_logits_adjust(lib.Logits(two[0::2]), two[1::2])
    assert torch.equal(two[1::2], two[0::2])
