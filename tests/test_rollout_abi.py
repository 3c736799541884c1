"""CPU-only checks of the token policy's operators: refusals on the host before any launch, struct layouts, and pins of the
fp64 checkers."""
import ctypes as C
import math
import os
import shutil
import subprocess

import numpy as np
import pytest
import torch

from oracle import rollout as ref
from paper_2512_15347_amd import binding as pg

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = C.CDLL(pg.LIB_PATH)
P = 4096                                                 # an address that nothing reads: calls are refused before a launch


def test_struct_sizes_are_the_compilers(tmp_path):
    gcc = shutil.which("gcc")
    if gcc is None:
        pytest.skip("no host C compiler")
    src = tmp_path / "abi.c"
    src.write_text('#include <stdio.h>\n#include "progrpo.h"\n'
                   'int main(void) { printf("%zu %zu %d\\n", sizeof(pg_cache), sizeof(pg_logits), PG_CACHE_MAX_ROWS); return 0; }\n')
    subprocess.check_call([gcc, "-std=c99", "-Wall", "-Wextra", "-pedantic", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o",
                           str(tmp_path / "abi")])
    out = subprocess.check_output([str(tmp_path / "abi")]).decode().split()
    assert [int(v) for v in out] == [C.sizeof(pg.pg_cache), C.sizeof(pg.pg_logits), pg.PG_CACHE_MAX_ROWS]


def cache(**change):
    c = pg.pg_cache(layers=2, n_pages=10, heads=4, page=16, head_dim=64, dtype=0, width=8, k=P, v=P, refs=P, status=P)
    for n, v in change.items():
        setattr(c, n, v)
    return C.byref(c)


BAD_CACHES = [(dict(layers=0), pg.PG_EINVAL), (dict(n_pages=0), pg.PG_EINVAL), (dict(heads=-1), pg.PG_EINVAL), (dict(width=0), pg.PG_EINVAL),
              (dict(dtype=2), pg.PG_EINVAL), (dict(page=8), pg.PG_ESHAPE), (dict(page=48), pg.PG_ESHAPE), (dict(head_dim=96), pg.PG_ESHAPE),
              (dict(width=1 << 27), pg.PG_ESHAPE), (dict(width=(1 << 26) + 1), pg.PG_ESHAPE), (dict(refs=None), pg.PG_EINVAL), (dict(status=None), pg.PG_EINVAL),
              (dict(refs=P + 4), pg.PG_ESHAPE), (dict(k_scale=P), pg.PG_EINVAL), (dict(k=None), pg.PG_EINVAL), (dict(v=P + 8), pg.PG_ESHAPE),
              (dict(heads=1 << 24), pg.PG_ESHAPE)]


@pytest.mark.parametrize("change,status", BAD_CACHES)
def test_bad_caches_are_refused_by_every_call(change, status):
    c = cache(**change)
    i = C.c_int64
    assert pg._lib.pg_cache_append(c, 0, P, P, 256, P, P, None, 1, 1, None) == status
    assert pg._lib.pg_cache_select(c, P, P, 1, P, P * 9, P * 9, 1, P, None) == status
    assert pg._lib.pg_cache_compact(c, P, P, 1, P, None) == status
    assert pg._lib.pg_paged_attention(c, 0, P, 256, P, 1, None, P, 1, 4, 0.0, 16, P, 256, None, None, 0, None) == status
    assert pg._lib.pg_paged_attention_workspace(c, 1, 4, 1 << 20) == 0
    if not {"k", "v"} & set(change):                         # these two calls need no data
        assert pg._lib.pg_cache_clear(c, None) == status
        assert pg._lib.pg_cache_reserve(c, P, P, P, P, 1, None) == status
        assert pg._lib.pg_cache_check(c, None) == status
    assert len(pg.pg_last_error()) > 10 and i(0).value == 0


def test_calls_on_the_cache_refuse_bad_arguments():
    c, f = cache(), pg._lib
    assert f.pg_cache_clear(None, None) == pg.PG_EINVAL
    assert f.pg_cache_reserve(c, P, P, P, P, -1, None) == pg.PG_EINVAL
    assert f.pg_cache_reserve(c, P, P, P, P, pg.PG_CACHE_MAX_ROWS + 1, None) == pg.PG_ESHAPE
    assert f.pg_cache_reserve(c, P, None, P, P, 1, None) == pg.PG_EINVAL
    assert f.pg_cache_reserve(c, None, None, None, None, 0, None) == pg.PG_OK
    for layer, stride, rows, tokens, k, cu, want in ((2, 256, 1, 1, P, None, pg.PG_EINVAL), (-1, 256, 1, 1, P, None, pg.PG_EINVAL),
                                                     (0, 255, 1, 1, P, None, pg.PG_ESHAPE), (0, 260, 1, 1, P, None, pg.PG_ESHAPE),
                                                     (0, 256, 1, 2, P, None, pg.PG_EINVAL), (0, 256, -1, 1, P, P, pg.PG_EINVAL),
                                                     (0, 256, 1, 1, P + 2, None, pg.PG_ESHAPE), (0, 256, 1, 1, None, None, pg.PG_EINVAL),
                                                     (0, 256, 1 << 23, 1, P, P, pg.PG_ESHAPE)):
        assert f.pg_cache_append(c, layer, k, P, stride, P, P, cu, rows, tokens, None) == want
    far = 1 << 20
    assert f.pg_cache_select(c, P, P, 1, P, far, far, pg.PG_CACHE_MAX_ROWS + 1, P, None) == pg.PG_ESHAPE
    assert f.pg_cache_select(c, P, P, -1, P, far, far, 1, P, None) == pg.PG_EINVAL
    assert f.pg_cache_select(c, P, P, 1, P, far, far, 1, None, None) == pg.PG_EINVAL
    assert f.pg_cache_select(c, P, P, 4, P, P + 32, far, 1, P, None) == pg.PG_EINVAL      # the tables overlap
    assert f.pg_cache_select(c, P, P, 4, P, far, P + 12, 1, P, None) == pg.PG_EINVAL      # the lengths overlap
    assert f.pg_cache_select(c, P, P, 4, far, far + 64, 2 * far, 17, P, None) == pg.PG_EINVAL      # src and the new table overlap
    assert f.pg_cache_select(c, P, P, 4, far, 2 * far, far + 4, 2, P, None) == pg.PG_EINVAL        # src and the new lengths
    assert f.pg_cache_select(c, P, P, 1, 2 * P, far, 2 * far, 1, P + 4, None) == pg.PG_ESHAPE
    assert f.pg_cache_compact(c, P, P, -1, P, None) == pg.PG_EINVAL
    assert f.pg_cache_compact(c, P, P, 1, None, None) == pg.PG_EINVAL
    assert f.pg_cache_scratch_ints(c, 100) >= 4 + 3 * 100 and f.pg_cache_scratch_ints(None, 3) == 0


def test_attention_refuses_bad_arguments():
    c, f = cache(), pg._lib

    def call(layer=0, q=P, qs=512, table=P, rows=3, row_of=None, lens=P, n=3, heads=8, scale=0.0, most=64, out=P, os_=512, ws=None, size=0, on=c):
        return f.pg_paged_attention(on, layer, q, qs, table, rows, row_of, lens, n, heads, scale, most, out, os_, None, ws, size, None)

    for change, want in ((dict(layer=2), pg.PG_EINVAL), (dict(q=None), pg.PG_EINVAL), (dict(qs=511), pg.PG_ESHAPE), (dict(qs=516), pg.PG_ESHAPE),
                         (dict(q=P + 2), pg.PG_ESHAPE), (dict(os_=504), pg.PG_ESHAPE), (dict(table=None), pg.PG_EINVAL), (dict(rows=2), pg.PG_EINVAL),
                         (dict(rows=0, row_of=P), pg.PG_EINVAL), (dict(lens=None), pg.PG_EINVAL), (dict(n=-1), pg.PG_EINVAL), (dict(heads=6), pg.PG_ESHAPE),
                         (dict(heads=0), pg.PG_EINVAL), (dict(scale=math.nan), pg.PG_EINVAL), (dict(scale=math.inf), pg.PG_EINVAL),
                         (dict(most=-1), pg.PG_EINVAL), (dict(out=None), pg.PG_EINVAL), (dict(n=0), pg.PG_OK)):
        assert call(**change) == want, change
    long = cache(width=1 << 20)
    need = f.pg_paged_attention_workspace(long, 1, 8, 1 << 20)
    assert need > 0
    one = dict(n=1, rows=1, most=1 << 20, on=long)
    assert call(**one) == pg.PG_EWORKSPACE and call(**one, ws=P, size=need - 1) == pg.PG_EWORKSPACE
    assert call(**one, ws=P + 4, size=need + 64) == pg.PG_ESHAPE
    assert "workspace" in pg.pg_last_error()


def logits(**change):
    d = pg.pg_logits(logits=P, stride=100, dtype=0, rows=3, vocab=100)
    for n, v in change.items():
        setattr(d, n, v)
    return C.byref(d)


@pytest.mark.parametrize("change,status", [
    (dict(rows=-1), pg.PG_EINVAL), (dict(vocab=0), pg.PG_EINVAL), (dict(dtype=2), pg.PG_EINVAL), (dict(logits=None), pg.PG_EINVAL),
    (dict(stride=99), pg.PG_EINVAL), (dict(logits=P + 2), pg.PG_ESHAPE), (dict(dtype=1, logits=P + 1), pg.PG_ESHAPE),
    (dict(tokens=P), pg.PG_EINVAL), (dict(repetition=P), pg.PG_EINVAL), (dict(bias_offsets=P, n_bias=2), pg.PG_EINVAL),
    (dict(bias_offsets=P, n_bias=-1), pg.PG_EINVAL), (dict(allow=P), pg.PG_EINVAL), (dict(allow=P, n_masks=2), pg.PG_EINVAL),
    (dict(vocab=(1 << 30) + 1, stride=1 << 31), pg.PG_ESHAPE)])
def test_bad_logits_are_refused(change, status):
    d = logits(**change)
    assert pg._lib.pg_logits_adjust(d, P, 100, None) == status
    assert pg._lib.pg_sample_tokens(d, None, 0, 0, None, P, P, P, None) == status


def test_calls_on_logits_refuse_bad_arguments():
    f = pg._lib
    assert f.pg_logits_adjust(None, P, 100, None) == pg.PG_EINVAL and f.pg_sample_tokens(None, None, 0, 0, None, P, P, P, None) == pg.PG_EINVAL
    assert f.pg_logits_adjust(logits(), None, 100, None) == pg.PG_EINVAL
    assert f.pg_logits_adjust(logits(), P * 5, 99, None) == pg.PG_ESHAPE and f.pg_logits_adjust(logits(), P + 1, 100, None) == pg.PG_ESHAPE
    assert f.pg_logits_adjust(logits(dtype=1), P, 100, None) == pg.PG_EINVAL            # in place: fp32 alone
    assert f.pg_logits_adjust(logits(), P, 101, None) == pg.PG_EINVAL                   # and of the same stride
    for i in range(3):
        p = [P, P, P]
        p[i] = None
        assert f.pg_sample_tokens(logits(), None, 0, 0, None, *p, None) == pg.PG_EINVAL
    assert f.pg_logits_adjust(logits(rows=0, logits=None), None, 0, None) == pg.PG_OK
    assert f.pg_sample_scratch_floats(0, 5) == 0 and f.pg_sample_scratch_floats(5, 0) == 0
    assert f.pg_sample_scratch_floats(3, 100000) > f.pg_sample_scratch_floats(3, 100) > 0


# ---------------------------------------------------------------- the checkers

def test_checkers_codes_are_torchs():
    v = ref.e4m3_values()
    want = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(v, want)
    x = np.concatenate([np.random.default_rng(0).standard_normal(5000) * 40, v[:127], (v[1:127] + v[:126]) / 2, [1e9, -1e9]])
    got = ref.to_e4m3(x.astype(np.float32))
    want = torch.from_numpy(x.astype(np.float32)).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    np.testing.assert_array_equal(got, want)


def test_checkers_attention_is_the_softmax():
    rng = np.random.default_rng(1)
    q, k, v = rng.standard_normal((6, 32)), rng.standard_normal((2, 9, 32)), rng.standard_normal((2, 9, 32))
    out, lse, _ = ref.attention(q, k, v, 0.4)
    for h in range(6):
        s = torch.from_numpy(k[h // 3] @ q[h] * 0.4)
        np.testing.assert_allclose(out[h], (torch.softmax(s, 0) @ torch.from_numpy(v[h // 3])).numpy(), rtol=1e-13)
        np.testing.assert_allclose(lse[h], float(torch.logsumexp(s, 0)), rtol=1e-13)


def test_checkers_pages_keep_every_sequence():
    """Whatever is forked, grown, dropped and moved, a row reads the tokens that its history wrote."""
    rng = np.random.default_rng(2)
    pages = ref.Pages(300, 16, 12)
    store, truth = {}, []

    def moved():
        for a, b in pages.moves:
            for i in range(16):
                if (a, i) in store:
                    store[b, i] = store[a, i]
        pages.moves.clear()

    pages.rows, pages.lens, truth = [[] for _ in range(4)], [0] * 4, [[] for _ in range(4)]
    for step in range(40):
        add = rng.integers(0, 9, size=len(pages.lens)).tolist() if len(pages.lens) < 20 else [1] * len(pages.lens)
        add = [a if n + a < 180 else 0 for a, n in zip(add, pages.lens)]
        pages.reserve(add)
        for r, m in enumerate(add):
            for i in range(pages.lens[r] - m, pages.lens[r]):
                store[pages.rows[r][i // 16], i % 16] = token = int(rng.integers(1 << 30))
                truth[r] = truth[r] + [token]
        if step % 3 == 2:
            src = rng.integers(-1, len(truth), size=int(rng.integers(3, 14))).tolist()
            pages.select(src)
            truth = [truth[s] if s >= 0 else [] for s in src]
        if step % 5 == 4:
            pages.compact()
            assert all(c == 0 for c in pages.refs[sum(c > 0 for c in pages.refs):])
        moved()
        for r, tokens in enumerate(truth):
            assert [store[pages.rows[r][i // 16], i % 16] for i in range(pages.lens[r])] == tokens
        held = [0] * 300
        for row in pages.rows:
            for p in row:
                held[p] += 1
        assert held == pages.refs
    assert pages.status == 0


def test_checkers_logits_by_hand():
    z = ref.adjusted([2.0, -2.0, 1.0, 0.5], [1, 3], [0, 0, 9], 2.0, 0.25, 0.125, [(2, 1.5), (2, 9.0)], np.array([True, True, True, False]))
    assert z.tolist() == [1.0 - 0.5 - 0.125, -4.0, 2.5, -math.inf]
    s, y = ref.scores(np.array([0.3, 0.2]), 0.0, 1, 2, 3)
    assert s.tolist() == y.tolist() == [0.3, 0.2]
    assert abs(ref.log_softmax_at(np.array([1.0, 1.0, -math.inf]), 1) + math.log(2)) < 1e-15


def test_more_workgroups_than_a_launch_has_room_for_are_refused():
    """2^24 workgroups of 256 lanes: what lies beyond 2^32 lanes would not run, without an error."""
    f = pg._lib
    wide = cache(heads=64, width=1 << 20)
    assert f.pg_cache_append(wide, 0, P, P, 64 * 64, P, P, P, 1 << 20, 1, None) == pg.PG_ESHAPE
    assert f.pg_paged_attention(cache(heads=512), 0, P, 512 * 64, P, 40000, None, P, 40000, 512, 0.0, 16, P, 512 * 64, None, None, 0, None) == pg.PG_ESHAPE
    assert f.pg_paged_attention(cache(), 0, P, 256, P, 70000, None, P, 70000, 4, 0.0, 16, P, 256, None, None, 0, None) == pg.PG_ESHAPE
    big = logits(rows=65535, vocab=1 << 20, stride=1 << 20)
    assert f.pg_logits_adjust(big, P, 1 << 20, None) == pg.PG_ESHAPE and f.pg_sample_tokens(big, None, 0, 0, None, P, P, P, None) == pg.PG_ESHAPE
    assert f.pg_logits_adjust(logits(rows=65536), P, 100, None) == pg.PG_ESHAPE
