"""Mask indices that no mask has."""
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
