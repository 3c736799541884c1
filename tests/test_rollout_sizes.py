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


def cache(heads, head_dim, dtype, width=1 << 16):
    import ctypes as C
    c = pg.pg_cache(layers=1, n_pages=10, heads=heads, page=16, head_dim=head_dim, dtype=dtype, width=width, k=4096, v=4096, refs=4096, status=4096)
    return C.byref(c)


@pytest.mark.parametrize("heads,group", [(1, 1), (8, 4), (12, 1), (2, 40), (300, 1)])
@pytest.mark.parametrize("head_dim,dtype", [(32, 0), (64, 1), (128, 0), (128, 1)])
def test_workspace_of_attention_does_not_shrink(heads, group, head_dim, dtype):
    """With more queries, or with longer ones."""
    c, f = cache(heads, head_dim, dtype), pg._lib.pg_paged_attention_workspace
    lengths = [0, 1, 100, 128, 129, 500, 768, 769, 1000, 1500, 1536, 1537, 2000, 2048, 2049, 3000, 4096, 10000, 65536, 1 << 20]
    rows = [r for r in ROWS if r * heads * (-(-group // 16)) < 1 << 24]
    for n in lengths:
        sizes = [f(c, r, heads * group, n) for r in rows]
        assert sizes == sorted(sizes), n
    for r in rows[::9] + [2048, 2049]:
        sizes = [f(c, r, heads * group, n) for n in lengths]
        assert sizes == sorted(sizes), r
    assert f(c, 0, heads * group, 1 << 20) == 0
