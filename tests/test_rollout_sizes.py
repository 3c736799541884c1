"""CPU-only: sizes that a program asks for once, for its largest call, hold for every smaller one (a prune makes calls smaller)."""
import pytest

from paper_2512_15347_amd import binding as pg

ROWS = sorted({1, 2, 3, 7, 48, 640, 700, 2049, 65535} | set(range(5, 3000, 37)) | {b + i for b in (256, 512, 1280, 2048, 4096) for i in (-1, 0, 1)})


@pytest.mark.parametrize("vocab", [1, 17, 2047, 2048, 2049, 4097, 32001, 65537, 131073, 1 << 20])
def test_scratch_of_a_draw_does_not_shrink_with_more_rows(vocab):
    sizes = [pg.pg_sample_scratch_floats(r, vocab) for r in ROWS]
    assert sizes == sorted(sizes) and sizes[0] >= 5
    assert max(sizes) <= 5 * (8192 + 65535)                  # 1.4 MB whatever the call


@pytest.mark.parametrize("rows", [1, 48, 384, 1280, 1281, 5000])
def test_scratch_of_a_draw_does_not_shrink_with_more_tokens(rows):
    sizes = [pg.pg_sample_scratch_floats(rows, v) for v in list(range(1, 200000, 997)) + [1 << 18, 1 << 22]]
    assert sizes == sorted(sizes)
