"""CPU-only: the binding takes tensors whose bits are what the kernels read them as, and no others."""
import pytest
import torch

from paper_2512_15347_amd import binding as pg


def pools(kind):
    return torch.zeros(1, 4, 2, 16, 64).to(kind), torch.zeros(1, 4, 2, 64, 16).to(kind), torch.zeros(4, dtype=torch.int32)


@pytest.mark.parametrize("kind,codes", [(torch.bfloat16, 0), (torch.int16, 0), (torch.uint16, 0), (torch.uint8, 1), (torch.int8, 1), (torch.float8_e4m3fn, 1)])
def test_pools_of_bf16_and_of_codes(kind, codes):
    assert pg.Cache(*pools(kind), 2).c.dtype == codes


@pytest.mark.parametrize("kind", [torch.float16, torch.float32, torch.float8_e5m2, torch.float8_e4m3fnuz, torch.bool])
def test_other_pools_are_refused(kind):
    with pytest.raises(AssertionError):
        pg.Cache(*pools(kind), 2)


def test_pools_of_two_kinds_are_refused():
    with pytest.raises(AssertionError):
        pg.Cache(pools(torch.bfloat16)[0], *pools(torch.float16)[1:], 2)


def test_queries_and_tokens_are_bf16():
    cache = pg.Cache(*pools(torch.bfloat16), 2)
    ints = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    x, half = (torch.zeros(3, 2, 64, dtype=k) for k in (torch.bfloat16, torch.float16))
    for q, out in ((half, x), (x, half), (half, half)):
        with pytest.raises(AssertionError):
            pg.pg_paged_attention(cache, 0, q, ints(3, 2), ints(3), out, 16)
    for k, v in ((half, x), (x, half)):
        with pytest.raises(AssertionError):
            pg.pg_cache_append(cache, 0, k, v, ints(3, 2), ints(3))


def test_scratch_of_draws_is_measured_in_bytes():
    d = pg.Logits(torch.zeros(3, 5000))
    token, logp = torch.zeros(3, dtype=torch.int32), torch.zeros(3)
    for kind, each in ((torch.uint8, 1), (torch.bfloat16, 2), (torch.float32, 4)):
        with pytest.raises(AssertionError):
            pg.pg_sample_tokens(d, None, 0, 0, None, token, logp, torch.zeros((d.scratch * 4 - 1) // each, dtype=kind), stream=0)
