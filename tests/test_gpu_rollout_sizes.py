"""Workspaces asked for once, for the largest call of a rollout, and used by all of its calls."""
import pytest
import torch

from test_gpu_rollout import DEV, say

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


def test_attention_stays_inside_the_workspace_of_the_largest_call(lib):
    """2049 queries are one workgroup each, fewer and longer ones are cut into ranges."""
    say("workspace of 2049 queries of 4096 tokens")
    g = torch.Generator(device=DEV).manual_seed(1)
    pool = lambda *s: torch.randn(s, device=DEV, generator=g).to(torch.bfloat16)  # noqa: E731
    cache = lib.Cache(pool(1, 256, 1, 16, 128), pool(1, 256, 1, 128, 16), torch.ones(256, dtype=torch.int32, device=DEV), 256)
    table = torch.arange(256, dtype=torch.int32, device=DEV)[None]
    most = 2049
    q, lens = pool(most, 2, 128), torch.arange(most, dtype=torch.int32, device=DEV) * 2
    out, row_of = torch.empty_like(q), torch.zeros(most, dtype=torch.int32, device=DEV)
    size = lib.pg_paged_attention_workspace(cache, most, 2, 4096)
    guard = torch.full((size // 4 + 4096,), 12345.0, device=DEV)
    first = None
    for rows in (most, 2048, 512, 9, 1):
        at = torch.arange(most - rows, most, device=DEV)                  # the longest ones
        lib.pg_paged_attention(cache, 0, q[at], table, lens[at], out[:rows], 4096, guard[:size // 4], row_of=row_of[:rows])
        assert (guard[size // 4:] == 12345.0).all(), rows
        first = out.clone() if first is None else first
        # the same sums cut in other places, both within (2^-15 + 2 far) max |v|, far = 4 hd 2^-24 sum |q k| / sqrt(hd) of scores in fp32 (sums up
        # to 12, values up to 6 here), and then within a bf16 of each other
        tol = 2 * (2.0 ** -15 + 2 * 4 * 128 * 2.0 ** -24 * 12) * 6
        assert ((out[:rows].float() - first[at].float()).abs() <= 2.0 ** -7 * first[at].float().abs() + tol).all(), rows
    lib.pg_cache_check(cache)


@pytest.mark.parametrize("heads,page,head_dim", [(65536, 128, 128), (2097151, 16, 32)])
def test_the_largest_pages_are_copied_and_moved(lib, heads, page, head_dim):
    """2^31 bytes, and the most that is less: a fork's copy, and a move."""
    say(f"pages of {heads * page * head_dim * 2} bytes")
    z = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device=DEV)  # noqa: E731
    cache = lib.Cache(z(1, 3, heads, page, head_dim), z(1, 3, heads, head_dim, page), torch.zeros(3, dtype=torch.int32, device=DEV), 1)
    lib.pg_cache_clear(cache)
    ints = lambda *v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    table, lens = torch.full((1, 1), -1, dtype=torch.int32, device=DEV), ints(0)
    lib.pg_cache_reserve(cache, table, lens, ints(5), lens)
    gen = torch.Generator(device=DEV).manual_seed(heads)
    for pool in (cache.k, cache.v):
        pool[0, 0].view(torch.int16).random_(-2 ** 15, 2 ** 15, generator=gen)
    scratch = torch.empty(lib.pg_cache_scratch_ints(cache, 2), dtype=torch.int32, device=DEV)
    two, lens_two, last, lens_last = (torch.empty(s, dtype=torch.int32, device=DEV) for s in ((2, 1), (2,), (1, 1), (1,)))
    lib.pg_cache_select(cache, table, lens, ints(0, 0), two, lens_two, scratch)
    lib.pg_cache_check(cache)
    same = lambda p, a, b: all(torch.equal(p[0, a, i::8].view(torch.int16), p[0, b, i::8].view(torch.int16)) for i in range(8))  # noqa: E731
    assert two.tolist() == [[0], [1]] and same(cache.k, 0, 1) and same(cache.v, 0, 1)
    lib.pg_cache_select(cache, two, lens_two, ints(1), last, lens_last, scratch)
    for pool in (cache.k, cache.v):
        pool[0, 0].zero_()
    lib.pg_cache_compact(cache, last, lens_last, scratch)
    lib.pg_cache_check(cache)
    assert last.tolist() == [[0]] and cache.refs.tolist() == [1, 0, 0] and same(cache.k, 0, 1) and same(cache.v, 0, 1)
    assert (cache.k[0, 0, -1].view(torch.int16) != 0).any() and (cache.k[0, 2, ::64] == 0).all()
