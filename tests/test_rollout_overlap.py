"""CPU-only: logits and what is written beside them."""
import ctypes as C

import pytest

from paper_2512_15347_amd import binding as pg

P = 1 << 20                                              # an address that nothing reads: calls are refused before a launch


@pytest.mark.parametrize("dtype,stride,out,out_stride", [
    (0, 100, P + 4, 100), (0, 100, P - 4, 100), (0, 100, P + 4 * 99, 100),                    # shifted by less than a row
    (0, 100, P + 4 * 2 * 100, 100), (0, 100, P - 4 * 2 * 100, 100),                           # the last row on the first
    (0, 250, P + 4 * 99, 250), (0, 250, P + 4 * (250 + 151), 250), (0, 250, P - 4 * (250 * 2 - 99), 250),      # ends of interleaved rows
    (0, 100, P + 4 * 40, 300), (0, 300, P + 4 * 350, 100), (0, 300, P - 4 * 290, 150),        # strides of two kinds
    (1, 100, P + 2 * 100, 100), (1, 400, P + 4 * 49, 200), (1, 110, P - 4 * 99, 1000)])
def test_rows_that_overlap_the_logits_are_refused(dtype, stride, out, out_stride):
    d = pg.pg_logits(logits=P, stride=stride, dtype=dtype, rows=3, vocab=100)
    assert pg._lib.pg_logits_adjust(C.byref(d), out, out_stride, None) == pg.PG_EINVAL
    assert "overlap" in pg.pg_last_error()
