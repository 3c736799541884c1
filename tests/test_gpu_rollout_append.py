"""New tokens into the cache: offsets that do not begin at 0, and rows that got no place."""
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


@pytest.mark.parametrize("new", [1, 9])
def test_a_row_without_a_place_leaves_shared_pages_as_they_are(lib, new):
    """Two rows share a whole page, the pool has a page for one of them only: reserve leaves the other as it is, and its token goes nowhere."""
    say(f"append of {new} after a reserve that was refused")
    for f8 in (False, True):
        b = lib.Cache.create(1, 2, 2, 16, 64, 4, dtype=lib.PG_CACHE_E4M3 if f8 else lib.PG_CACHE_BF16)
        lib.pg_cache_clear(b)
        rng = np.random.default_rng(new)
        draw = lambda n: bf16(rng.standard_normal((n, 2, 64))).to(DEV)  # noqa: E731
        table, lens = torch.full((1, 4), -1, dtype=torch.int32, device=DEV), dev([0])
        lib.pg_cache_reserve(b, table, lens, dev([16]), lens)
        lib.pg_cache_append(b, 0, draw(16), draw(16), table, lens, cu=dev([0, 16]))
        two, lens_two = torch.empty(2, 4, dtype=torch.int32, device=DEV), torch.empty(2, dtype=torch.int32, device=DEV)
        scratch = torch.empty(lib.pg_cache_scratch_ints(b, 2), dtype=torch.int32, device=DEV)
        lib.pg_cache_select(b, table, lens, dev([0, 0]), two, lens_two, scratch)
        assert b.refs.tolist() == [2, 0]
        lib.pg_cache_reserve(b, two, lens_two, dev([new, new]), lens_two)
        assert lens_two.tolist() == [16 + new, 16] and int(b.status[0]) == 4
        before = b.k[0, 0].clone(), b.v[0, 0].clone()
        k, v = draw(2 * new), draw(2 * new)
        lib.pg_cache_append(b, 0, k, v, two, lens_two, cu=None if new == 1 else dev([0, new, 2 * new]))
        assert torch.equal(b.k[0, 0].view(torch.uint8), before[0].view(torch.uint8)) and torch.equal(b.v[0, 0].view(torch.uint8), before[1].view(torch.uint8))
        if not f8:
            assert torch.equal(b.k[0, 1, :, :new].transpose(0, 1), k[:new]) and torch.equal(b.v[0, 1, :, :, :new].permute(2, 0, 1), v[:new])
        with pytest.raises(lib.PgError) as e:
            lib.pg_cache_check(b)
        assert e.value.status == lib.PG_EWORKSPACE
