"""CPU-only: factors that 32 bits do not hold."""
import ctypes as C

import pytest

from paper_2512_15347_amd import binding as pg

P = 4096


@pytest.mark.parametrize("scale", [1e39, -1e39, 3.4e38, 1e300])
def test_a_scale_past_the_largest_float_is_refused(scale):
    """Logits are kept in base 2, so the factor is log2(e) times the scale; as a float it is infinite for all of these."""
    c = pg.pg_cache(layers=1, n_pages=10, heads=4, page=16, head_dim=64, dtype=0, width=8, k=P, v=P, refs=P, status=P)
    assert pg._lib.pg_paged_attention(C.byref(c), 0, P, 256, P, 1, None, P, 1, 4, scale, 16, P, 256, None, None, 0, None) == pg.PG_EINVAL
