"""GPU parity of the token policy's operators against plain fp64 checkers, through the C ABI."""
import math

import numpy as np
import pytest
import torch

from oracle import rollout as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U24 = 2.0 ** -24


def say(msg):
    print(msg, flush=True)


def dev(a, dtype=np.int32):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=dtype)).to(DEV)


def bf16(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(torch.bfloat16)


# ------------------------------------------------------------------ attention over pages

def make_cache(lib, rng, lens, kv, hd, page, f8, shared=0, layers=1, spread=0):
    """A cache whose unused slots hold NaN, its table, and what each row's tokens are in fp64."""
    pages = [-(-n // page) for n in lens]
    whole = shared // page
    n_pages = sum(pages) + 3 + spread
    order = rng.permutation(n_pages)
    if spread:                                       # page numbers from the far end of a large pool
        order = np.concatenate([np.arange(n_pages - sum(pages) - 3, n_pages)])
        rng.shuffle(order)
    width = max(pages + [1]) + 1
    table = np.full((len(lens), width), -1, dtype=np.int32)
    refs = np.zeros(n_pages, dtype=np.int32)
    at = whole
    for r, n in enumerate(pages):
        own = order[at:at + max(0, n - whole)]
        at += len(own)
        row = np.concatenate([order[:min(whole, n)], own])
        table[r, :n] = row
        refs[row] += 1
    scales = None
    if f8:
        scales = rng.uniform(0.01, 0.05, size=(2, layers, kv)).astype(np.float32)
    dtype = torch.uint8 if f8 else torch.bfloat16
    k = torch.full((layers, n_pages, kv, page, hd), 0x7F, dtype=dtype, device=DEV) if f8 else \
        torch.full((layers, n_pages, kv, page, hd), float("nan"), dtype=dtype, device=DEV)
    v = k.reshape(layers, n_pages, kv, hd, page).clone()
    cache = lib.Cache(k, v, dev(refs), width, *(() if not f8 else (dev(scales[0], np.float32), dev(scales[1], np.float32))))
    values = ref.e4m3_values()
    filled = {}
    for r, n in enumerate(lens):                     # tokens of every page that is not yet filled, in the last layer
        for j in range(pages[r]):
            p, m = int(table[r, j]), min(page, n - j * page)
            if p in filled and filled[p][0].shape[1] >= m:
                continue
            x = rng.standard_normal((2, kv, page, hd)).astype(np.float32)
            if f8:
                codes = ref.to_e4m3(x * 16)
                x = values[codes] * scales[:, -1, :, None, None]
                kb, vb = (torch.from_numpy(c) for c in codes)
            else:
                kb, vb = bf16(x[0]), bf16(x[1])
                x = np.stack([kb.float().numpy(), vb.float().numpy()]).astype(np.float64)
            cache.k[-1, p, :, :m] = kb[:, :m].to(DEV)
            cache.v[-1, p, :, :, :m] = vb[:, :m].transpose(1, 2).to(DEV)
            filled[p] = (x[0, :, :m], x[1, :, :m])
    rows = []
    for r, n in enumerate(lens):
        empty = [np.zeros((kv, 0, hd))] * 2
        rows.append([np.concatenate([e] + [filled[int(p)][i] for p in table[r, :pages[r]]], axis=1)[:, :n] for i, e in enumerate(empty)])
    return cache, dev(table), rows


def check_attention(lib, rng, cache, table, rows, lens, heads, hd, max_len, row_of=None, scale=0.0, sharp=1.0, stream=None, pad=0, layer=0):
    n_q = len(lens)
    wide = torch.full((n_q, heads + pad, hd), float("nan"), dtype=torch.bfloat16, device=DEV)
    q = wide[:, :heads]
    q.copy_(bf16(rng.standard_normal((n_q, heads, hd)) * sharp))
    out = torch.full((n_q, heads + pad, hd), float("nan"), dtype=torch.bfloat16, device=DEV)
    lse = torch.full((n_q, heads), float("nan"), device=DEV)
    ws = torch.empty(max(16, lib.pg_paged_attention_workspace(cache, n_q, heads, max_len)), dtype=torch.uint8, device=DEV)
    torch.cuda.synchronize()
    lib.pg_paged_attention(cache, layer, q, table, dev(lens), out[:, :heads], max_len, ws, lse=lse,
                           row_of=None if row_of is None else dev(row_of), scale=scale, stream=stream)
    torch.cuda.synchronize()
    lib.pg_cache_check(cache)
    qn, got, got_lse = q.float().cpu().numpy().astype(np.float64), out.float().cpu().numpy(), lse.cpu().numpy()
    assert np.isnan(got[:, heads:]).all()
    for i, n in enumerate(lens):
        k, v = rows[i if row_of is None else row_of[i]]
        k, v = k[:, :n], v[:, :n]
        want, want_lse, size = ref.attention(qn[i], k, v, scale or 1 / math.sqrt(hd))
        # scores summed in fp32 (hd terms, and two factors more), probabilities kept to 17 bits, 32-bit sums: what is then rounded to
        # bf16 is no further off than tol, and the rounding is monotonic
        far = 4 * hd * U24 * max(size, 1.0)
        tol = (2.0 ** -15 + 2 * far) * (np.abs(v).max() if n else 0.0)
        lo, hi = (torch.from_numpy(b).to(torch.bfloat16).float().numpy() for b in (want - tol, want + tol))
        assert ((lo <= got[i, :heads]) & (got[i, :heads] <= hi)).all(), (i, n, np.max(np.maximum(lo - got[i, :heads], got[i, :heads] - hi)))
        if n == 0:
            assert (got[i, :heads] == 0).all() and (got_lse[i] == -np.inf).all()
        else:
            assert (np.abs(got_lse[i] - want_lse) <= far + 8 * U24 * (np.abs(want_lse) + 1)).all(), (i, n)
    return out


LENGTHS = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 200, 511, 513]


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("hd", [32, 64, 128])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
def test_attention_at_every_edge_of_pages_and_steps(lib, page, hd, f8):
    say(f"paged attention, page {page}, head width {hd}, {'codes' if f8 else 'bf16'}")
    rng = np.random.default_rng([page, hd, f8])
    cache, table, rows = make_cache(lib, rng, LENGTHS, 2, hd, page, f8)
    check_attention(lib, rng, cache, table, rows, LENGTHS, 6, hd, 513, pad=5)
    check_attention(lib, rng, cache, table, rows, LENGTHS, 2, hd, 513, scale=0.3)
    check_attention(lib, rng, cache, table, rows, LENGTHS, 8, hd, 1, sharp=6.0)        # longer than said: right all the same


@pytest.mark.parametrize("kv,group", [(1, 1), (3, 1), (1, 16), (2, 17), (1, 48), (5, 7)])
def test_attention_head_layouts(lib, kv, group):
    say(f"paged attention, {kv} key/value heads of {group} query heads")
    rng = np.random.default_rng([kv, group])
    lens = [77, 1, 300]
    for f8 in (False, True):
        cache, table, rows = make_cache(lib, rng, lens, kv, 64, 16, f8)
        check_attention(lib, rng, cache, table, rows, lens, kv * group, 64, 300)


@pytest.mark.parametrize("n,f8", [(5000, False), (9001, True)])
def test_attention_split_over_a_long_row(lib, n, f8):
    say(f"paged attention over {n} tokens")
    rng = np.random.default_rng(n)
    for lens in ([n], [n, 3, 0, n // 2]):
        cache, table, rows = make_cache(lib, rng, lens, 2, 128, 64, f8)
        check_attention(lib, rng, cache, table, rows, lens, 8, 128, n)
        check_attention(lib, rng, cache, table, rows, lens, 8, 128, n, sharp=8.0)


@pytest.mark.parametrize("rows,kv,group,hd,page,f8", [(30, 4, 3, 64, 16, False), (23, 3, 20, 128, 64, False), (17, 5, 2, 128, 32, True), (40, 2, 4, 32, 16, True)])
def test_attention_in_even_ranges(lib, rows, kv, group, hd, page, f8):
    """More units than ranges, so that a range covers several rows, some whole; empty rows at both ends and between; two tiles of heads."""
    say(f"paged attention in even ranges: {rows} rows, {kv} x {group} heads of {hd}")
    rng = np.random.default_rng([rows, kv, hd])
    lens = rng.integers(1, 5000, size=rows)
    lens[[0, 5, 6, rows - 1]] = 0
    lens[7] = 9000
    lens = lens.tolist()
    cache, table, rows_ = make_cache(lib, rng, lens, kv, hd, page, f8)
    assert lib.pg_paged_attention_workspace(cache, rows, kv * group, 9000) > 0
    check_attention(lib, rng, cache, table, rows_, lens, kv * group, hd, 9000, sharp=2.0)


def test_a_row_longer_than_said_and_than_the_page_numbers_in_lds(lib):
    say("paged attention, 20000 tokens in pages of 16 by one workgroup")
    rng = np.random.default_rng(12)
    lens = [20000, 8192, 8193]
    cache, table, rows = make_cache(lib, rng, lens, 1, 32, 16, False)
    check_attention(lib, rng, cache, table, rows, lens, 2, 32, 1)
    check_attention(lib, rng, cache, table, rows, lens, 2, 32, 20000)


def test_attention_of_a_prompt_as_queries_of_growing_lengths(lib):
    """Rows of the table in any order and repeated; pages shared by several rows; the last of two layers."""
    say("paged attention with a row map")
    rng = np.random.default_rng(5)
    cache, table, rows = make_cache(lib, rng, [70, 66, 90], 2, 64, 16, False, shared=64, layers=2)
    row_of = [0] * 70 + [2, 1, 1, 2]
    lens = list(range(1, 71)) + [90, 66, 5, 0]
    check_attention(lib, rng, cache, table, rows, lens, 4, 64, 90, row_of=row_of, layer=1)


def test_attention_on_another_stream_and_in_a_graph(lib):
    say("paged attention on a side stream, and replayed")
    rng = np.random.default_rng(6)
    lens = [300, 40, 1500]
    cache, table, rows = make_cache(lib, rng, lens, 2, 64, 16, False)
    side = torch.cuda.Stream()
    check_attention(lib, rng, cache, table, rows, lens, 8, 64, 1500, stream=side)
    q = bf16(rng.standard_normal((3, 8, 64))).to(DEV)
    out, lse = torch.zeros(3, 8, 64, dtype=torch.bfloat16, device=DEV), torch.zeros(3, 8, device=DEV)
    ws = torch.empty(max(16, lib.pg_paged_attention_workspace(cache, 3, 8, 1500)), dtype=torch.uint8, device=DEV)
    d = dev(lens)
    call = lambda: lib.pg_paged_attention(cache, 0, q, table, d, out, 1500, ws, lse=lse)  # noqa: E731
    call()
    torch.cuda.synchronize()
    want, want_lse = out.clone(), lse.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for _ in range(4):
        out.zero_()
        lse.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(lse, want_lse)
        call()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(lse, want_lse)


def test_pages_beyond_32_bit_offsets(lib):
    """A pool of more than 2^31 elements: attention, append and fork on its last pages."""
    say("pages beyond 2^31 elements")
    rng = np.random.default_rng(7)
    lens = [130, 257]
    cache, table, rows = make_cache(lib, rng, lens, 8, 128, 128, False, spread=17000)
    assert cache.k.numel() > 2 ** 31
    check_attention(lib, rng, cache, table, rows, lens, 8, 128, 257)
    k, v = (bf16(rng.standard_normal((2, 8, 128))).to(DEV) for _ in range(2))
    lib.pg_cache_append(cache, 0, k, v, table, dev(lens))
    for i, n in enumerate(lens):
        p = int(table[i, (n - 1) // 128])
        assert torch.equal(cache.k[0, p, :, (n - 1) % 128], k[i]) and torch.equal(cache.v[0, p, :, :, (n - 1) % 128], v[i])
    cache.refs[:-8] = 1                              # only pages at the far end are free
    new, lens_new = torch.zeros(4, table.shape[1], dtype=torch.int32, device=DEV), torch.zeros(4, dtype=torch.int32, device=DEV)
    scratch = torch.empty(lib.pg_cache_scratch_ints(cache, 4), dtype=torch.int32, device=DEV)
    lib.pg_cache_select(cache, table, dev(lens), dev([0, 1, 1, 0]), new, lens_new, scratch)
    lib.pg_cache_check(cache)
    assert int(new[2, 2]) != int(new[1, 2]) and int(new[2, 2]) > 17000 - 8 and int(new[3, 1]) != int(new[0, 1])
    valid = (257 - 1) % 128 + 1
    assert torch.equal(cache.k[0, int(new[2, 2]), :, :valid], cache.k[0, int(new[1, 2]), :, :valid])
    assert torch.equal(cache.v[0, int(new[2, 2]), :, :, :valid], cache.v[0, int(new[1, 2]), :, :, :valid])


def test_attention_flags_what_lies_outside_the_table(lib):
    rng = np.random.default_rng(8)
    cache, table, rows = make_cache(lib, rng, [40, 20], 1, 64, 16, False)
    q, out = torch.zeros(2, 1, 64, dtype=torch.bfloat16, device=DEV), torch.ones(2, 1, 64, dtype=torch.bfloat16, device=DEV)
    for lens, row_of, t in (([40, 10 ** 6], None, table), ([-1, 20], None, table), ([40, 20], [0, 7], table), ([40, 20], None, table + 1000)):
        cache.status.zero_()
        lib.pg_paged_attention(cache, 0, q, t, dev(lens), out, 40, None, row_of=None if row_of is None else dev(row_of))
        with pytest.raises(lib.PgError) as e:
            lib.pg_cache_check(cache)
        assert e.value.status == lib.PG_EINVAL


# ------------------------------------------------------------------ new tokens into the cache

@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("hd,page,kv", [(32, 16, 1), (64, 16, 3), (64, 128, 5), (128, 32, 8), (128, 64, 2)])
def test_append_writes_the_new_tokens_and_nothing_else(lib, hd, page, kv, f8):
    say(f"append, head width {hd}, page {page}, {kv} heads, {'codes' if f8 else 'bf16'}")
    rng = np.random.default_rng([hd, page, kv, f8])
    lens = [1, 16, 17, 100, 0, 33, 250, 64, 5] + [19] * 70
    for new in ([1] * len(lens), [min(n, m) for n, m in zip(lens, [1, 16, 3, 100, 0, 0, 131, 40, 5] + list(range(70)))]):
        if new == [1] * len(lens):
            lens = [max(1, n) for n in lens]
        cache, table, _ = make_cache(lib, rng, lens, kv, hd, page, f8, layers=2)
        k0, v0 = cache.k.cpu().clone(), cache.v.cpu().clone()
        T = sum(new)
        x = rng.standard_normal((T, 2 * kv + 1, hd)) * 2
        x.reshape(-1)[:6] = [np.nan, 1e30, -1e30, 0.0, -0.0, 1e-30]
        wide = bf16(x).to(DEV)
        kn, vn = wide[:, :kv], wide[:, kv:2 * kv]
        cu = np.concatenate([[0], np.cumsum(new)])
        one_each = new == [1] * len(lens)
        lib.pg_cache_append(cache, 1, kn, vn, table, dev(lens), cu=None if one_each else dev(cu))
        lib.pg_cache_check(cache)
        t = table.cpu().numpy()
        codes = lambda a, s: torch.from_numpy(ref.to_e4m3((a.float() / s[1].cpu()[:, None]).numpy())) if f8 else a  # noqa: E731
        kc, vc = codes(kn.cpu(), cache.k_scale), codes(vn.cpu(), cache.v_scale)
        for r, n in enumerate(lens):
            for i in range(new[r]):
                at = n - new[r] + i
                p = int(t[r, at // page])
                k0[1, p, :, at % page] = kc[cu[r] + i]
                v0[1, p, :, :, at % page] = vc[cu[r] + i]
        as_int = lambda a: a.view(torch.uint8) if f8 else a.view(torch.int16)  # noqa: E731
        for got, want in ((cache.k, k0), (cache.v, v0)):
            same = as_int(got.cpu()) == as_int(want)
            if f8:
                same |= (as_int(got.cpu()) & 0x7F == 0x7F) & (as_int(want) & 0x7F == 0x7F)      # either NaN
            assert same.all()


def test_append_flags_counts_that_do_not_fit(lib):
    rng = np.random.default_rng(3)
    cache, table, _ = make_cache(lib, rng, [20, 30], 1, 64, 16, False)
    x = torch.zeros(6, 1, 64, dtype=torch.bfloat16, device=DEV)
    for lens, cu in (([20, 30], [0, 2, 7]), ([2, 30], [0, 4, 6]), ([20, 10 ** 6], [0, 3, 6]), ([20, 30], [4, 2, 6]), ([20, 30], [-3, 2, 6])):
        cache.status.zero_()
        before = cache.refs.clone()
        lib.pg_cache_append(cache, 0, x, x, table, dev(lens), cu=dev(cu))
        with pytest.raises(lib.PgError) as e:
            lib.pg_cache_check(cache)
        assert e.value.status == lib.PG_EINVAL and torch.equal(before, cache.refs)


def test_every_code_round_trips_and_ties_go_to_even(lib):
    say("e4m3 rounding")
    v = ref.e4m3_values()[:127]
    x = np.concatenate([v, (v[1:] + v[:-1]) / 2, (v[1:] + v[:-1]) / 2 * (1 + 2.0 ** -7), [449, 1e4, np.inf]])
    x = np.concatenate([x, -x])
    x = np.concatenate([x, np.zeros(-len(x) % 64)]).reshape(-1, 1, 64)
    xb = bf16(x)
    n = len(x)
    cache = lib.Cache.create(1, -(-n // 16), 1, 16, 64, -(-n // 16), dtype=lib.PG_CACHE_E4M3)
    table = torch.arange(-(-n // 16), dtype=torch.int32, device=DEV)[None]
    lib.pg_cache_append(cache, 0, xb.to(DEV), xb.to(DEV), table, dev([n]), cu=dev([0, n]))
    got = cache.k[0, :, 0].reshape(-1, 64)[:n].cpu().numpy()
    want = ref.to_e4m3(xb.float().numpy()[:, 0])
    np.testing.assert_array_equal(got, want)
    np.testing.assert_array_equal(want, xb.float().clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8).numpy()[:, 0])


def test_codes_are_those_of_the_rounded_quotient_for_every_bf16_and_any_scale(lib):
    say("e4m3 codes of all 65536 patterns")
    scales = np.array([1.0, 3.0, 1 / 3, 0.0173, 0.7, 1.9999999, 1.0000001, 448.0, 1e-3, 7e4, 1e30, 3e38, 1e-30, 1.2e-38, 1e-38, 2e-39, 1e-40, 1e-45,
                       0.0625, 5.5, 11.0, 0.3, 123.456, 0.99999994], dtype=np.float32).reshape(3, 8)
    bits = torch.arange(65536, dtype=torch.int32).to(torch.int16)
    x = bits.view(torch.bfloat16).reshape(1024, 1, 64).expand(-1, 8, -1).contiguous()
    cache = lib.Cache.create(3, 64, 8, 16, 64, 64, dtype=lib.PG_CACHE_E4M3)
    cache.k_scale.copy_(torch.from_numpy(scales))
    cache.v_scale.copy_(torch.from_numpy(scales))
    table = torch.arange(64, dtype=torch.int32, device=DEV)[None]
    for layer in range(3):
        lib.pg_cache_append(cache, layer, x.to(DEV), x.to(DEV), table, dev([1024]), cu=dev([0, 1024]))
        k = cache.k[layer].permute(1, 0, 2, 3).reshape(8, 65536).cpu().numpy()
        v = cache.v[layer].permute(1, 0, 3, 2).reshape(8, 65536).cpu().numpy()
        for h in range(8):
            with np.errstate(all="ignore"):
                want = ref.to_e4m3(x[:, h].reshape(-1).float().numpy() / scales[layer, h])
            nan = want & 0x7F == 0x7F
            for got in (k[h], v[h]):
                assert ((got & 0x7F == 0x7F) == nan).all() and (got[~nan] == want[~nan]).all(), (scales[layer, h], np.flatnonzero((got != want) & ~nan)[:5])


# ------------------------------------------------------------------ pages

class Both:
    """The library's pages beside the checker's."""

    def __init__(self, lib, n_pages, page, width, layers=2, kv=2, hd=32):
        self.lib, self.model = lib, ref.Pages(n_pages, page, width)
        self.cache = lib.Cache.create(layers, n_pages, kv, page, hd, width)
        lib.pg_cache_clear(self.cache)
        g = torch.Generator(device=DEV).manual_seed(n_pages)
        for pool in (self.cache.k, self.cache.v):
            pool.view(torch.int16).random_(-2 ** 15, 2 ** 15, generator=g)
        self.k, self.v = self.cache.k.view(torch.int16).cpu().clone(), self.cache.v.view(torch.int16).cpu().clone()
        self.table = torch.full((0, width), -1, dtype=torch.int32, device=DEV)
        self.lens = torch.zeros(0, dtype=torch.int32, device=DEV)

    def rows(self, n):
        self.model.rows, self.model.lens = [[] for _ in range(n)], [0] * n
        self.table = torch.full((n, self.model.width), -1, dtype=torch.int32, device=DEV)
        self.lens = torch.zeros(n, dtype=torch.int32, device=DEV)

    def reserve(self, add):
        self.model.reserve(add)
        self.lib.pg_cache_reserve(self.cache, self.table, self.lens, dev(add), self.lens)
        self.same()

    def select(self, src):
        self.model.select(src)
        n = max(len(src), self.table.shape[0])
        scratch = torch.full((self.lib.pg_cache_scratch_ints(self.cache, n),), -7, dtype=torch.int32, device=DEV)
        table = torch.full((len(src), self.model.width), 99, dtype=torch.int32, device=DEV)
        lens = torch.full((len(src),), 99, dtype=torch.int32, device=DEV)
        self.lib.pg_cache_select(self.cache, self.table, self.lens, dev(src), table, lens, scratch)
        self.table, self.lens = table, lens
        self.same()

    def compact(self):
        self.model.compact()
        scratch = torch.full((self.lib.pg_cache_scratch_ints(self.cache, 0),), -7, dtype=torch.int32, device=DEV)
        self.lib.pg_cache_compact(self.cache, self.table, self.lens, scratch)
        self.same()

    def same(self):
        torch.cuda.synchronize()
        assert self.lens.cpu().tolist() == self.model.lens
        assert self.cache.refs.cpu().tolist() == self.model.refs
        np.testing.assert_array_equal(self.table.cpu().numpy(), self.model.table())
        assert int(self.cache.status[0]) == self.model.status
        for a, b in self.model.moves:
            self.k[:, b], self.v[:, b] = self.k[:, a], self.v[:, a]
        self.model.moves.clear()
        assert torch.equal(self.cache.k.view(torch.int16).cpu(), self.k) and torch.equal(self.cache.v.view(torch.int16).cpu(), self.v)


@pytest.mark.parametrize("page,n_pages", [(16, 400), (32, 203), (64, 129), (128, 64)])
def test_a_groups_pages_from_prompt_to_survivors(lib, page, n_pages):
    say(f"pages of {page}: expand, grow, prune, compact")
    rng = np.random.default_rng(page)
    b = Both(lib, n_pages, page, 12)
    b.rows(3)
    b.reserve([3 * page, 2 * page + 5, 1])
    b.select([0] * 5 + [1] * 6 + [2] * 7)                # whole pages shared, part-filled ones copied
    for _ in range(3):
        b.reserve(rng.integers(0, page, size=18).tolist())
    keep = sorted(rng.choice(18, size=7, replace=False).tolist())
    b.select(keep)
    b.compact()
    b.reserve([page + 3] * 7)
    b.select([6, 0, 0, -1, 3])
    b.compact()
    b.select([-1, -1])
    assert sum(b.model.refs) == 0
    b.select([])
    b.rows(2)
    b.reserve([0, 7])
    assert b.model.status == 0


def test_random_lives_of_pages(lib):
    """Sequences of calls with empty rows, exhausted pools, full tables and bad sources."""
    for seed in range(6):
        rng = np.random.default_rng([11, seed])
        b = Both(lib, int(rng.integers(3, 60)), 16, int(rng.integers(2, 6)), layers=1, kv=1)
        b.rows(int(rng.integers(1, 9)))
        say(f"random life {seed}: {len(b.model.refs)} pages")
        for _ in range(12):
            n, what = len(b.model.lens), rng.integers(0, 4)
            if what == 0 and n:
                b.reserve([int(v) for v in rng.integers(-1 if rng.random() < 0.2 else 0, 40, size=n)])
            elif what == 1:
                b.compact()
            else:
                b.select([int(v) for v in rng.integers(-2 if rng.random() < 0.2 else -1, max(1, n) + (rng.random() < 0.1), size=int(rng.integers(1, 12)))])
            b.cache.status.zero_()
            b.model.status = 0


def test_as_many_rows_as_a_call_takes(lib):
    say("16384 rows")
    n = lib.PG_CACHE_MAX_ROWS
    b = Both(lib, 3 * n, 16, 3, layers=1, kv=1)
    b.rows(n)
    b.reserve([(r * 7) % 33 for r in range(n)])
    b.select([(r * 3) % (n // 2) for r in range(n)])
    b.reserve([r % 2 for r in range(n)])
    b.compact()


def test_reserve_in_order_until_the_pool_ends(lib):
    b = Both(lib, 5, 16, 4)
    b.rows(4)
    b.reserve([16, 40, 48, 0])                           # one, three, none of three
    assert b.model.lens == [16, 40, 0, 0] and b.model.status == 4
    with pytest.raises(lib.PgError) as e:
        lib.pg_cache_check(b.cache)
    assert e.value.status == lib.PG_EWORKSPACE
    b.reserve([0, 8, 16, 1])                             # inside the page that is there; the last page; none
    assert b.model.lens == [16, 48, 16, 0]
    b.reserve([70, 0, 0, 0])                             # wider than the table
    assert b.model.lens[0] == 16


# ------------------------------------------------------------------ logits

def logits_case(rng, R, V, dtype, H=0, masks=0, bias=0, scale=3.0):
    x = rng.standard_normal((R, V + 3)) * scale
    t = torch.from_numpy(x.astype(np.float32)).to(dtype).to(DEV)[:, 1:V + 1]      # rows of longer ones, off any alignment
    rows = dict(x=t.float().cpu().numpy().astype(np.float64), prompt=[[]] * R, output=[[]] * R, rep=[1.0] * R, freq=[0.0] * R, pres=[0.0] * R,
                bias=[[]] * R, allowed=[None] * R)
    more = {}
    f32 = lambda a: np.asarray(a, dtype=np.float32)  # noqa: E731
    if H:
        tok = np.where(rng.random((R, H)) < 0.5, rng.integers(-2, min(V + 2, 12), size=(R, H)), rng.integers(0, V, size=(R, H))).astype(np.int32)
        n = rng.integers(0, H + 1, size=R)
        n[0] = H
        m = np.minimum(n, rng.integers(0, H + 1, size=R))
        rep, freq, pres = f32(rng.uniform(0.8, 1.5, R)), f32(rng.uniform(-0.2, 0.5, R)), f32(rng.uniform(0, 0.7, R))
        more = dict(tokens=dev(tok), n_prompt=dev(m), n_tokens=dev(n), repetition=dev(rep, np.float32), frequency=dev(freq, np.float32),
                    presence=dev(pres, np.float32))
        rows.update(prompt=[tok[r, :m[r]] for r in range(R)], output=[tok[r, m[r]:n[r]] for r in range(R)], rep=rep.astype(np.float64),
                    freq=freq.astype(np.float64), pres=pres.astype(np.float64))
    if masks:
        words = (V + 31) // 32
        a = rng.integers(0, 2 ** 32, size=(masks, words), dtype=np.uint32)
        a[-1] = 0
        which = rng.integers(-1, masks, size=R).astype(np.int32)
        more.update(allow=dev(a.view(np.int32)), allow_row=dev(which))
        bits = (a[:, np.arange(V) // 32] >> (np.arange(V) % 32).astype(np.uint32) & 1).astype(bool)
        rows["allowed"] = [bits[w] if w >= 0 else None for w in which]
    if bias:
        offs, ids, vals = [0], [], []
        for r in range(R):
            k = int(rng.integers(0, bias + 1))
            ids += sorted(rng.integers(0, V, size=k).tolist())
            vals += f32(rng.standard_normal(k) * 4).tolist()
            offs.append(len(ids))
        rows["bias"] = [list(zip(ids[offs[r]:offs[r + 1]], vals[offs[r]:offs[r + 1]])) for r in range(R)]
        more.update(bias_offsets=dev(offs), bias_ids=dev(ids + [0]), bias_values=dev(vals + [0.0], np.float32))
    return t, more, rows


def adjusted_rows(rows):
    return [ref.adjusted(*(rows[n][r] for n in ("x", "prompt", "output", "rep", "freq", "pres", "bias", "allowed"))) for r in range(len(rows["x"]))]


CASES = [(1, 1, 0, 0, 0), (3, 7, 5, 1, 3), (5, 1000, 40, 3, 20), (2, 2047, 0, 2, 0), (2, 2049, 300, 0, 0), (4, 32001, 1178, 2, 64), (40, 65537, 64, 4, 300),
         (12, 4099, 2500, 2, 4000), (3, 9000, 20000, 0, 500)]      # nearly every token has both; a history longer than what stays in registers


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("R,V,H,masks,bias", CASES)
def test_adjusted_logits(lib, R, V, H, masks, bias, dtype):
    say(f"adjust {R} x {V}, history {H}, {masks} masks, lists of {bias}, {dtype}")
    rng = np.random.default_rng([R, V, H])
    t, more, rows = logits_case(rng, R, V, dtype, H, masks, bias)
    wide = torch.full((R, V + 5), 77.0, device=DEV)
    lib.pg_logits_adjust(lib.Logits(t, **more), wide[:, 3:V + 3])
    got = wide.cpu().numpy().astype(np.float64)
    assert (got[:, :3] == 77).all() and (got[:, V + 3:] == 77).all()
    for r, z in enumerate(adjusted_rows(rows)):
        g = got[r, 3:V + 3]
        np.testing.assert_array_equal(np.isneginf(g), np.isneginf(z))
        fine = np.isfinite(z)
        # five roundings of values no larger than the logit, its penalties and its bias
        size = np.abs(rows["x"][r]) * 2 + 0.7 + 0.5 * H + 40
        assert (np.abs(g[fine] - z[fine]) <= 5 * U24 * size[fine]).all()
    if dtype == torch.float32:                           # in place
        lib.pg_logits_adjust(lib.Logits(t, **more), t)
        assert torch.equal(t, wide[:, 3:V + 3])


def test_adjusted_logits_pass_nan_and_infinity_of_masked_places_over(lib):
    x = torch.tensor([[float("nan"), 1.0, float("inf"), 2.0, -float("inf")]], device=DEV)
    allow = dev([[0b01010]])
    out = torch.empty_like(x)
    lib.pg_logits_adjust(lib.Logits(x, allow=allow), out)
    assert out.tolist() == [[-math.inf, 1.0, -math.inf, 2.0, -math.inf]]
    token, logp = torch.zeros(1, dtype=torch.int32, device=DEV), torch.zeros(1, device=DEV)
    scratch = torch.empty(lib.pg_sample_scratch_floats(1, 5), device=DEV)
    lib.pg_sample_tokens(lib.Logits(x, allow=allow), None, 1, 0, None, token, logp, scratch)
    assert int(token) in (1, 3)
    assert abs(float(logp) - (-math.log1p(math.exp(1.0)) + (1.0 if int(token) == 3 else 0.0))) < 1e-5


# ------------------------------------------------------------------ draws

@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("R,V,H,masks,bias", CASES)
def test_drawn_tokens_and_log_probs(lib, R, V, H, masks, bias, dtype):
    say(f"sample {R} x {V}, history {H}, {masks} masks, lists of {bias}, {dtype}")
    rng = np.random.default_rng([R, V, H, 1])
    t, more, rows = logits_case(rng, R, V, dtype, H, masks, bias)
    T = np.asarray(rng.uniform(0.5, 1.5, R), dtype=np.float32)
    T[1::3] = 0.0
    ids = rng.integers(0, 2 ** 31, size=R).astype(np.int32)
    seed, step = 0xFEDCBA9876543210, 12345
    token, logp = torch.full((R,), -5, dtype=torch.int32, device=DEV), torch.full((R,), 5.0, device=DEV)
    scratch = torch.full((lib.pg_sample_scratch_floats(R, V),), float("nan"), device=DEV)
    lib.pg_sample_tokens(lib.Logits(t, **more), dev(T, np.float32), seed, step, dev(ids), token, logp, scratch)
    again = token.clone(), logp.clone()
    lib.pg_sample_tokens(lib.Logits(t, **more), dev(T, np.float32), seed, step, dev(ids), token, logp, scratch)
    assert torch.equal(again[0], token) and torch.equal(again[1], logp)
    for r, z in enumerate(adjusted_rows(rows)):
        got, lp = int(token[r]), float(logp[r])
        if not np.isfinite(z).any():
            assert got == -1 and lp == -math.inf
            continue
        score, y = ref.scores(z, float(T[r]), seed, step, int(ids[r]))
        size = np.abs(y[np.isfinite(y)]).max() + 30 + 0.5 * H
        # scores and log-probs in fp32: some ten roundings of values up to `size`
        assert score[got] >= score.max() - 16 * U24 * size, (r, got, int(score.argmax()))
        assert abs(lp - ref.log_softmax_at(y, got)) <= 16 * U24 * size


@pytest.mark.parametrize("R", [60, 380, 800, 1400])
def test_a_draw_does_not_depend_on_the_rows_beside_it(lib, R):
    """Rows of one stretch a workgroup, of two, whole ones, and more rows than are resident: each draws what it draws in a call of seven."""
    say(f"draws of {R} rows")
    rng = np.random.default_rng(R)
    V, H = 24001, 300
    t, more, rows = logits_case(rng, 7, V, torch.float32, H, 2)
    T = torch.tensor([1.0, 0.0, 0.7, 1.3, 1.0, 1.0, 0.9], device=DEV)
    at = torch.arange(R, device=DEV) % 7
    one, one_p, many, many_p = (torch.full((n,), -5, dtype=k, device=DEV) for n in (7, R) for k in (torch.int32, torch.float32))
    scratch = torch.empty(max(lib.pg_sample_scratch_floats(n, V) for n in (7, R)), device=DEV)
    ids = torch.arange(7, dtype=torch.int32, device=DEV) * 11
    lib.pg_sample_tokens(lib.Logits(t, **more), T, 5, 9, ids, one, one_p, scratch)
    wide = {n: x if n == "allow" else x[at].contiguous() for n, x in more.items()}
    lib.pg_sample_tokens(lib.Logits(t[at].contiguous(), **wide), T[at], 5, 9, ids[at], many, many_p, scratch)
    assert torch.equal(many, one[at])                    # a token's score is its own
    # each log-prob is within some ten roundings of values up to `size`, as above; sums are taken in another order
    size = max(np.abs(z[np.isfinite(z)]).max(initial=0.0) for z in adjusted_rows(rows)) / 0.7 + 30 + 0.5 * H
    assert ((many_p == one_p[at]) | ((many_p - one_p[at]).abs() <= 32 * U24 * size)).all()


def test_draws_follow_the_softmax_and_the_ids(lib):
    say("draws' frequencies")
    R, V = 20000, 17
    rng = np.random.default_rng(2)
    row = rng.standard_normal(V) * 1.5
    x = torch.from_numpy(np.tile(row, (R, 1)).astype(np.float32)).to(DEV)
    ids = torch.randperm(R, device=DEV).to(torch.int32)
    token, logp = torch.zeros(R, dtype=torch.int32, device=DEV), torch.zeros(R, device=DEV)
    scratch = torch.empty(lib.pg_sample_scratch_floats(R, V), device=DEV)
    lib.pg_sample_tokens(lib.Logits(x), None, 99, 3, ids, token, logp, scratch)
    p = np.exp(row - row.max())
    p /= p.sum()
    n = np.bincount(token.cpu().numpy(), minlength=V)
    chi2 = float(((n - R * p) ** 2 / (R * p)).sum())
    assert chi2 < 45.0                                   # 16 degrees of freedom: exceeded once in 7000
    # the same ids in another order draw the same tokens
    other, order = torch.zeros_like(token), torch.argsort(ids)
    lib.pg_sample_tokens(lib.Logits(x), None, 99, 3, None, other, logp, scratch)
    assert torch.equal(token[order], other)
    lib.pg_sample_tokens(lib.Logits(x), None, 99, 4, None, other, logp, scratch)
    assert not torch.equal(token[order], other)


def test_rows_that_cannot_be_drawn_from(lib):
    nan, inf = float("nan"), float("inf")
    x = torch.zeros(9, 40, device=DEV)
    x[0, 3], x[1, 39], x[2] = nan, inf, -inf
    x[3, :39] = -inf
    t = dev([1, 1, 1, 1, -1, nan, inf, 0, 1], np.float32)
    x[7, 5] = x[7, 21] = 4.0                             # equal ones: the lowest
    x[8, :] = -3e38
    token, logp = torch.zeros(9, dtype=torch.int32, device=DEV), torch.zeros(9, device=DEV)
    lib.pg_sample_tokens(lib.Logits(x), t, 5, 0, None, token, logp, torch.empty(lib.pg_sample_scratch_floats(9, 40), device=DEV))
    token, logp = token.tolist(), logp.tolist()
    assert token[:7] == [-1, -1, -1, 39, -1, -1, -1] and token[7] == 5
    assert all(math.isnan(logp[i]) for i in (0, 1, 4, 5, 6)) and logp[2] == -inf and logp[3] == 0.0
    assert 0 <= token[8] < 40 and abs(logp[8] + math.log(40)) < 1e-5


def test_nothing_to_do(lib):
    e = lambda *s, dtype=torch.int32: torch.empty(*s, dtype=dtype, device=DEV)  # noqa: E731
    cache = lib.Cache.create(1, 4, 1, 16, 64, 2)
    lib.pg_cache_reserve(cache, e(0, 2), e(0), e(0), e(0))
    x = e(0, 1, 64, dtype=torch.bfloat16)
    lib.pg_cache_append(cache, 0, x, x, e(0, 2), e(0))
    lib.pg_paged_attention(cache, 0, x, e(1, 2), e(0), x.clone(), 5)
    lib.pg_cache_select(cache, e(0, 2), e(0), e(0), e(0, 2), e(0), e(100))
    lib.pg_cache_compact(cache, e(0, 2), e(0), e(100))
    z = e(0, 9, dtype=torch.float32)
    lib.pg_logits_adjust(lib.Logits(z), z)
    lib.pg_sample_tokens(lib.Logits(z), None, 0, 0, None, e(0), e(0, dtype=torch.float32), e(0, dtype=torch.float32))
    lib.pg_cache_check(cache)
