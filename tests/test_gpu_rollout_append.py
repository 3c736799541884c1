"""New tokens into the cache: offsets that do not begin at 0."""
import numpy as np
import pytest
import torch

from test_gpu_rollout import DEV, bf16, dev, make_cache, say

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("start", [1, 15, 16, 17, 40, 1000])
def test_offsets_may_begin_anywhere(lib, start):
    say(f"append from token {start} on")
    rng = np.random.default_rng(start)
    lens, new = [30, 7, 64, 0, 19], [17, 7, 64, 0, 1]
    for f8 in (False, True):
        cache, table, _ = make_cache(lib, rng, lens, 2, 64, 16, f8)
        cu = start + np.concatenate([[0], np.cumsum(new)])
        k, v = (bf16(rng.standard_normal((int(cu[-1]), 2, 64))).to(DEV) for _ in range(2))
        lib.pg_cache_append(cache, 0, k, v, table, dev(lens), cu=dev(cu))
        lib.pg_cache_check(cache)
        again = lib.Cache(torch.zeros_like(cache.k), torch.zeros_like(cache.v), cache.refs, cache.width, cache.k_scale, cache.v_scale)
        for c in (cache, again):                            # what lies beside the new tokens, cleared
            for r, n in enumerate(lens):
                for j in range(-(-n // 16)):
                    p, lo, hi = int(table[r, j]), max(0, n - new[r] - 16 * j), min(16, n - 16 * j)
                    for pool, at in ((c.k[0, p], 1), (c.v[0, p], 2)):
                        pool.narrow(at, 0, max(0, min(lo, 16))).zero_()
                        pool.narrow(at, hi, 16 - hi).zero_()
        lib.pg_cache_append(again, 0, k[start:], v[start:], table, dev(lens), cu=dev(cu - start))
        lib.pg_cache_check(again)
        used = torch.unique(table[table >= 0]).long()
        same = lambda a, b: torch.equal(a[0, used].view(torch.uint8), b[0, used].view(torch.uint8))  # noqa: E731
        assert same(cache.k, again.k) and same(cache.v, again.v)
