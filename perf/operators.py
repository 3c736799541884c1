"""The operators of an autoregressive policy's rollouts, as their users call them: for timing, and for comparing the kernels
with their plain forms.

Five kinds of work:
  attend   attention of one new token of each sequence over a paged key/value cache (pg_paged_attention)
  append   keys and values of new tokens into the cache's pages (pg_cache_append)
  pages    the life of a group's pages: expand, reserve, prune (pg_cache_select, pg_cache_reserve), or compaction (pg_cache_compact)
  adjust   penalties, biases and grammar masks on logits (pg_logits_adjust)
  sample   the same, a draw from the softmax and the drawn token's log-prob (pg_sample_tokens)

The cache: K [layers, pages, heads, page, head_dim], V [layers, pages, heads, head_dim, page] (values transposed), bf16 or 8-bit
e4m3 codes with a scale for each layer and head; a table [rows, width] of page numbers (-1: none) and a length for each row; a
reference count for each page (0: free).  Lengths follow from the case alone, values from the seed.
"""
import functools
import math

import torch

own = False
DEV = "cuda:0"
FP8_MAX = 448.0


def listed():
    return [
        # ---- attention ----
        # one short sequence of a small network (12 heads of 64, the 77 tokens of a prompt): latency alone
        dict(name="attend_one", work="attend", rows=1, lo=77, hi=77, heads=12, kv_heads=12, hd=64, page=16, dtype="bf16", shared=0),
        # a group of 48 in the middle of its rollout: 154 prompt tokens that all share, up to 1024 tokens of its own
        dict(name="attend_group", work="attend", rows=48, lo=155, hi=1178, heads=24, kv_heads=8, hd=64, page=16, dtype="bf16", shared=154),
        # eight groups of 48 with ragged lengths from one token on, a cache of 8-bit codes, pages of 64
        dict(name="attend_batch", work="attend", rows=384, lo=1, hi=4096, heads=32, kv_heads=8, hd=128, page=64, dtype="e4m3", shared=0),
        # three very long sequences: all of the work is split over the length
        dict(name="attend_long", work="attend", rows=3, lo=65537, hi=131071, heads=32, kv_heads=4, hd=128, page=128, dtype="bf16", shared=0),
        # ---- new tokens into the cache ----
        # one token for each of a group of 48
        dict(name="append_token", work="append", rows=48, lo=155, hi=1178, new=1, kv_heads=8, hd=64, page=16, dtype="bf16"),
        # prompts of all lengths from one token on, rounded to 8 bits
        dict(name="append_prompts", work="append", rows=64, lo=1, hi=4097, new=0, kv_heads=8, hd=128, page=32, dtype="e4m3"),
        # ---- pages ----
        # 8 prompts expanded to 48 members each, a token's place for each member, pruned to 16 of 48
        dict(name="expand_and_prune", work="pages", what="funnel", groups=8, members=48, keep=16, lo=77, hi=1178, kv_heads=8, hd=64, page=16,
             layers=12),
        # a pool after many prunes: live pages scattered, moved together
        dict(name="compact_pool", work="pages", what="compact", rows=150, lo=33, hi=2049, live=0.6, kv_heads=8, hd=128, page=64, layers=2),
        # ---- logits ----
        # a group of 48 over a codebook of 16384 tokens
        dict(name="adjust_codebook", work="adjust", rows=48, vocab=16384, dtype="f32", history=1178, masks=4, bias=32),
        # eight groups of 48 over an odd vocabulary
        dict(name="adjust_text", work="adjust", rows=384, vocab=65537, dtype="bf16", history=2048, masks=16, bias=300),
        # one row, nothing but the draw: latency
        dict(name="sample_one", work="sample", rows=1, vocab=32001, dtype="f32", history=0, masks=0, bias=0),
        # eight groups of 48 over a large vocabulary with all adjustments
        dict(name="sample_batch", work="sample", rows=384, vocab=131073, dtype="bf16", history=1178, masks=16, bias=32),
    ]


def draw(rng):
    def log_int(lo, hi):
        return min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)) - 0.5 / hi))) or 1)

    work = rng.choice(["attend", "attend", "append", "pages", "adjust", "sample"])
    if work == "attend":
        kv = rng.choice([1, 2, 4, 8, 12])
        c = dict(work=work, rows=log_int(1, 400), heads=kv * rng.choice([1, 2, 3, 4, 8, 16]), kv_heads=kv, hd=rng.choice([64, 128]),
                 page=rng.choice([16, 32, 64, 128]), dtype=rng.choice(["bf16", "e4m3"]), shared=0)
        most = 131071
        while c["rows"] * most * kv * c["hd"] * (2 if c["dtype"] == "bf16" else 1) > 2 ** 28:
            most = most * 3 // 4
        c["hi"] = log_int(min(16, most), most)
        c["lo"] = log_int(1, c["hi"])
        if rng.random() < 0.3:
            c["shared"] = c["lo"] - 1
        return c
    if work == "append":
        hd, new = rng.choice([64, 128]), rng.choice([0, 1, 1, 5])
        hi = log_int(8, 4097)
        return dict(work=work, rows=log_int(1, 64 if new == 0 else 256), lo=min(hi, 5 + log_int(1, hi)), hi=hi, new=new, kv_heads=rng.choice([1, 2, 4, 8]), hd=hd,
                    page=rng.choice([16, 32, 64, 128]), dtype=rng.choice(["bf16", "e4m3"]))
    if work == "pages":
        c = dict(work=work, kv_heads=rng.choice([1, 2, 4, 8]), hd=rng.choice([64, 128]), page=rng.choice([16, 32, 64]))
        if rng.random() < 0.5:
            members = log_int(2, 48)
            hi = log_int(8, 1178)
            return dict(c, what="funnel", groups=log_int(1, 8), members=members, keep=rng.randint(1, members), lo=log_int(1, hi), hi=hi,
                        layers=log_int(1, 12) if c["page"] * c["hd"] <= 2048 else 1)
        hi = log_int(16, 2049)
        return dict(c, what="compact", rows=log_int(1, 150), lo=log_int(1, hi), hi=hi, live=rng.choice([0.3, 0.6, 0.9]), layers=rng.choice([1, 2]))
    rows = log_int(1, 384)
    return dict(work=work, rows=rows, vocab=log_int(1000, 131073 if work == "sample" else 65537), dtype=rng.choice(["f32", "bf16"]),
                history=rng.choice([0, log_int(1, 2048)]), masks=rng.choice([0, 1, 16]), bias=rng.choice([0, 1, 300]))


# ---------------------------------------------------------------- what a user's program has in hand

def _lengths(rows, lo, hi):
    """Lengths between lo and hi, spread evenly in a scattered order; the first row has the longest."""
    return [hi if r == 0 else lo + int(((r * 0.6180339887498949) % 1.0) * (hi - lo + 1)) for r in range(rows)]


def _pages(n, page):
    return -(-n // page)


def _tables(lengths, page, shared, rng, spare=1.1, width=0):
    """Tables over a pool in random order; the whole pages of the first `shared` tokens are the same ones for every row."""
    whole = shared // page
    need = whole + sum(_pages(n, page) - min(whole, n // page) for n in lengths)
    n_pages = max(need + 1, int(need * spare))
    order = torch.randperm(n_pages, generator=rng).tolist()
    width = max([width] + [_pages(n, page) for n in lengths])
    table = torch.full((len(lengths), width), -1, dtype=torch.int32)
    refs = torch.zeros(n_pages, dtype=torch.int32)
    at = whole
    for r, n in enumerate(lengths):
        own_pages = _pages(n, page) - min(whole, n // page)
        row = order[:min(whole, n // page)] + order[at:at + own_pages]
        at += own_pages
        table[r, :len(row)] = torch.tensor(row, dtype=torch.int32)
        refs[row] += 1
    return table.to(DEV), refs.to(DEV), n_pages


def _pool(layers, n_pages, kv, page, hd, dtype, gen):
    """K and V pools, and their scales where they hold codes."""
    out = []
    for shape in ((layers, n_pages, kv, page, hd), (layers, n_pages, kv, hd, page)):
        if dtype == "bf16":
            out.append(torch.empty(shape, dtype=torch.bfloat16, device=DEV).normal_(generator=gen))
        else:
            codes = torch.empty(shape, dtype=torch.uint8, device=DEV)
            step = max(1, (1 << 26) // (kv * page * hd))
            for lay in range(layers):
                for p in range(0, n_pages, step):
                    part = codes[lay, p:p + step]
                    part.copy_((torch.randn(part.shape, device=DEV, generator=gen) * 32).to(torch.float8_e4m3fn).view(torch.uint8))
            out.append(codes)
    scales = [None, None]
    if dtype != "bf16":
        scales = [torch.rand(layers, kv, device=DEV, generator=gen) / 64 + 1 / 64 for _ in range(2)]
    return dict(k=out[0], v=out[1], k_scale=scales[0], v_scale=scales[1])


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    host = torch.Generator().manual_seed(seed)
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    s = dict(case=case)
    if case["work"] == "attend":
        lengths = _lengths(case["rows"], case["lo"], case["hi"])
        s["table"], s["refs"], n_pages = _tables(lengths, case["page"], case["shared"], host)
        s.update(_pool(1, n_pages, case["kv_heads"], case["page"], case["hd"], case["dtype"], gen))
        s["lens"] = ints(lengths)
        # queries come as the first columns of the projection of queries, keys and values; twice the unit size gives the few
        # large weights that softmax rows have
        wide = torch.randn(case["rows"], case["heads"] + 2 * case["kv_heads"], case["hd"], device=DEV, generator=gen) * 2
        s["q"] = wide.to(torch.bfloat16)[:, :case["heads"]]
        s["out"] = torch.empty(case["rows"], case["heads"], case["hd"], dtype=torch.bfloat16, device=DEV)
        s["lse"] = torch.empty(case["rows"], case["heads"], device=DEV)
    elif case["work"] == "append":
        lengths = _lengths(case["rows"], case["lo"], case["hi"])
        new = [min(n, case["new"] or n) for n in lengths]
        s["table"], s["refs"], n_pages = _tables(lengths, case["page"], 0, host)
        s.update(_pool(1, n_pages, case["kv_heads"], case["page"], case["hd"], case["dtype"], gen))
        s["lens"] = ints(lengths)
        s["cu"] = ints([sum(new[:r]) for r in range(len(new) + 1)]) if case["new"] != 1 else None
        wide = torch.randn(sum(new), 4 * case["kv_heads"], case["hd"], device=DEV, generator=gen).to(torch.bfloat16)
        s["k_new"], s["v_new"] = wide[:, 2 * case["kv_heads"]:3 * case["kv_heads"]], wide[:, 3 * case["kv_heads"]:]
    elif case.get("what") == "funnel":
        P, N, k = case["groups"], case["members"], case["keep"]
        lengths = _lengths(P, case["lo"], case["hi"])
        page = case["page"]
        spare = 1 + 2.0 * P * N / (sum(_pages(n, page) for n in lengths))
        s["table"], s["refs0"], n_pages = _tables(lengths, page, 0, host, spare, width=_pages(case["hi"] + 1, page))
        s["refs"] = s["refs0"].clone()
        s.update(_pool(case["layers"], n_pages, case["kv_heads"], page, case["hd"], "bf16", gen))
        s["lens"] = ints(lengths)
        s["expand"] = ints([g for g in range(P) for _ in range(N)])
        s["ones"] = torch.ones(P * N, dtype=torch.int32, device=DEV)
        kept = [g * N + i for g in range(P) for i in sorted(torch.randperm(N, generator=host)[:k].tolist())]
        s["prune"] = ints(kept)
        width = s["table"].shape[1]
        for name, rows in (("many", P * N), ("few", P * k)):
            s["table_" + name] = torch.empty(rows, width, dtype=torch.int32, device=DEV)
            s["lens_" + name] = torch.empty(rows, dtype=torch.int32, device=DEV)
        s["lens_grown"] = torch.empty(P * N, dtype=torch.int32, device=DEV)
    elif case.get("what") == "compact":
        lengths = _lengths(case["rows"], case["lo"], case["hi"])
        s["table0"], s["refs0"], n_pages = _tables(lengths, case["page"], 0, host, 1 / case["live"])
        s["table"], s["refs"] = s["table0"].clone(), s["refs0"].clone()
        s.update(_pool(case["layers"], n_pages, case["kv_heads"], case["page"], case["hd"], "bf16", gen))
        s["lens"] = ints(lengths)
    else:
        R, V, H = case["rows"], case["vocab"], case["history"]
        x = torch.randn(R, V, device=DEV, generator=gen) * 3
        s["logits"] = x if case["dtype"] == "f32" else x.to(torch.bfloat16)
        s["tokens"] = s["allow"] = s["bias_ids"] = None
        if H:
            # a few tokens come often, most hardly ever; rows are filled to different lengths, the first third is the prompt
            u = torch.rand(R, H, device=DEV, generator=gen)
            s["tokens"] = (V * u * u * u).to(torch.int32)
            n = _lengths(R, 1, H)
            s["n_tokens"], s["n_prompt"] = ints(n), ints([v // 3 for v in n])
            s["repetition"] = 1 + 0.3 * torch.rand(R, device=DEV, generator=gen)
            s["frequency"] = 0.2 * torch.rand(R, device=DEV, generator=gen)
            s["presence"] = 0.5 * torch.rand(R, device=DEV, generator=gen)
        if case["masks"]:
            m, words = case["masks"], _pages(V, 32)
            a = torch.randint(-2 ** 31, 2 ** 31, (m, words), device=DEV, generator=gen).to(torch.int32)
            # half of the masks leave runs of tokens out, as a grammar does, and of more than one the last allows nothing
            a[1::2] |= torch.randint(-2 ** 31, 2 ** 31, a[1::2].shape, device=DEV, generator=gen).to(torch.int32)
            if m > 1:
                a[m - 1] = 0
            s["allow"] = a
            rows = torch.randint(-1, max(1, m - 1), (R,), generator=host)
            if m > 1 and R > 8:
                rows[5] = m - 1
            s["allow_row"] = rows.to(torch.int32).to(DEV)
        if case["bias"]:
            ids, offsets = [], [0]
            for r in range(R):
                n = min(V, (r * 7) % (case["bias"] + 1))
                ids.append(torch.sort(torch.randperm(V, generator=host)[:n] if n > 64 else torch.unique(torch.randint(0, V, (n,), generator=host)))[0])
                offsets.append(offsets[-1] + ids[-1].numel())
            s["bias_offsets"] = ints(offsets)
            s["bias_ids"] = torch.cat(ids + [torch.zeros(1, dtype=torch.int64)]).to(torch.int32).to(DEV)
            s["bias_values"] = torch.randn(s["bias_ids"].shape, device=DEV, generator=gen) * 4
        if case["work"] == "adjust":
            s["out"] = torch.empty(R, V, device=DEV)
        else:
            t = 0.7 + 0.6 * torch.rand(R, device=DEV, generator=gen)
            t[3::16] = 0.0                                  # some rows take the most likely token
            s["temperature"] = t
            s["ids"] = torch.randperm(4 * R, generator=host)[:R].to(torch.int32).to(DEV)
            s["key"], s["step"] = (seed * 0x9E3779B97F4A7C15 + 77) & (2 ** 64 - 1), seed % 1000
            s["token"] = torch.empty(R, dtype=torch.int32, device=DEV)
            s["logp"] = torch.empty(R, device=DEV)
    return s


def work(case):
    if case["work"] == "attend":
        lengths = _lengths(case["rows"], case["lo"], case["hi"])
        whole = case["shared"] // case["page"] * case["page"]
        once = whole + sum(n - min(whole, n // case["page"] * case["page"]) for n in lengths)      # shared pages count once
        elt = 2 if case["dtype"] == "bf16" else 1
        per_row = case["heads"] * (4 * case["hd"] + 4) + 4
        return dict(bytes=2 * once * case["kv_heads"] * case["hd"] * elt + case["rows"] * per_row + 4 * sum(_pages(n, case["page"]) for n in lengths),
                    flops=4 * sum(lengths) * case["heads"] * case["hd"])
    if case["work"] == "append":
        new = sum(min(n, case["new"] or n) for n in _lengths(case["rows"], case["lo"], case["hi"]))
        return dict(bytes=2 * new * case["kv_heads"] * case["hd"] * (2 + (2 if case["dtype"] == "bf16" else 1)), flops=0)
    if case["work"] == "pages":
        page_bytes = 4 * case["kv_heads"] * case["page"] * case["hd"] * case["layers"]
        if case["what"] == "funnel":
            lengths, page = _lengths(case["groups"], case["lo"], case["hi"]), case["page"]
            copies = sum(case["members"] - 1 for n in lengths if n % page)
            width = _pages(case["hi"] + 1, page)
            rows = case["groups"] * (1 + 2 * case["members"] + case["keep"])
            return dict(bytes=2 * copies * page_bytes + 4 * rows * width, flops=0)
        lengths = _lengths(case["rows"], case["lo"], case["hi"])
        live = sum(_pages(n, case["page"]) for n in lengths)
        n_pages = max(live + 1, int(live / case["live"]))
        return dict(bytes=2 * live * (n_pages - live) / n_pages * page_bytes + 8 * live, flops=0)
    R, V = case["rows"], case["vocab"]
    read = R * V * (4 if case["dtype"] == "f32" else 2) + 4 * sum(_lengths(R, 1, case["history"]) if case["history"] else [0])
    read += case["masks"] * _pages(V, 32) * 4 + R * case["bias"] * 4
    if case["work"] == "adjust":
        return dict(bytes=read + 4 * R * V, flops=4 * R * V)
    return dict(bytes=read + 8 * R, flops=36 * R * V)


# ---------------------------------------------------------------- one pass

def run(s):
    return (_own if own else _plain)[s["case"]["work"]](s)


# ---- the framework's calls

def _cache(s):
    """The handle that a program keeps beside its pools."""
    from paper_2512_15347_amd import binding as pg
    if "cache" not in s:
        s["cache"] = pg.Cache(s["k"], s["v"], s["refs"], s["table"].shape[1], k_scale=s["k_scale"], v_scale=s["v_scale"])
    return pg, s["cache"]


def _own_attend(s):
    pg, cache = _cache(s)
    if "workspace" not in s:
        s["workspace"] = torch.empty(pg.pg_paged_attention_workspace(cache, s["case"]["rows"], s["case"]["heads"], s["case"]["hi"]), dtype=torch.uint8,
                                     device=DEV)
    pg.pg_paged_attention(cache, 0, s["q"], s["table"], s["lens"], s["out"], s["case"]["hi"], s["workspace"], lse=s["lse"])
    return dict(out=s["out"], lse=s["lse"])


def _own_append(s):
    pg, cache = _cache(s)
    pg.pg_cache_append(cache, 0, s["k_new"], s["v_new"], s["table"], s["lens"], cu=s["cu"])
    return _pools(s)


def _pools(s):
    values = (lambda t: t) if s["k_scale"] is None else (lambda t: t.view(torch.float8_e4m3fn))
    return dict(k=values(s["k"]), v=values(s["v"]))


def _own_pages(s):
    pg, cache = _cache(s)
    if "scratch" not in s:
        rows = max(s["case"].get("groups", 0) * s["case"].get("members", 0), s["table"].shape[0])
        s["scratch"] = torch.empty(pg.pg_cache_scratch_ints(cache, rows), dtype=torch.int32, device=DEV)
    s["refs"].copy_(s["refs0"])
    if s["case"]["what"] == "compact":
        s["table"].copy_(s["table0"])
        pg.pg_cache_compact(cache, s["table"], s["lens"], s["scratch"])
        return dict(table=s["table"], refs=s["refs"], **_pools(s))
    pg.pg_cache_select(cache, s["table"], s["lens"], s["expand"], s["table_many"], s["lens_many"], s["scratch"])
    pg.pg_cache_reserve(cache, s["table_many"], s["lens_many"], s["ones"], s["lens_grown"])
    pg.pg_cache_select(cache, s["table_many"], s["lens_grown"], s["prune"], s["table_few"], s["lens_few"], s["scratch"])
    return dict(many=s["table_many"], lens_many=s["lens_grown"], few=s["table_few"], lens_few=s["lens_few"], refs=s["refs"], **_pools(s))


def _descriptor(s):
    from paper_2512_15347_amd import binding as pg
    if "descriptor" not in s:
        more = {}
        if s["tokens"] is not None:
            more.update({n: s[n] for n in ("tokens", "n_prompt", "n_tokens", "repetition", "frequency", "presence")})
        if s["allow"] is not None:
            more.update(allow=s["allow"], allow_row=s["allow_row"])
        if s["bias_ids"] is not None:
            more.update({n: s[n] for n in ("bias_offsets", "bias_ids", "bias_values")})
        s["descriptor"] = pg.Logits(s["logits"], **more)
    return pg, s["descriptor"]


def _own_adjust(s):
    pg, d = _descriptor(s)
    pg.pg_logits_adjust(d, s["out"])
    return s["out"]


def _own_sample(s):
    pg, d = _descriptor(s)
    if "scratch" not in s:
        s["scratch"] = torch.empty(pg.pg_sample_scratch_floats(s["case"]["rows"], s["case"]["vocab"]), device=DEV)
    pg.pg_sample_tokens(d, s["temperature"], s["key"], s["step"], s["ids"], s["token"], s["logp"], s["scratch"])
    return dict(token=s["token"], logp=s["logp"])


# ---- the plain forms

def _gathered(s, name):
    """The pages of every row, [rows, heads, tokens, hd] in 32 bits."""
    pages = s[name][0][s["table"].clamp_min(0).long()]                       # [rows, pages, heads, ., .]
    if name == "v":
        pages = pages.transpose(3, 4)
    x = pages.transpose(1, 2).flatten(2, 3)
    if s["k_scale"] is None:
        return x.float()
    return x.contiguous().view(torch.float8_e4m3fn).float() * s[name + "_scale"][0][:, None, None]


def _plain_attend(s):
    c = s["case"]
    q = s["q"].float().reshape(c["rows"], c["kv_heads"], -1, c["hd"])
    k = _gathered(s, "k")
    there = (torch.arange(k.shape[2], device=DEV) < s["lens"][:, None])[:, None, None]
    x = torch.matmul(q, k.transpose(2, 3)) / math.sqrt(c["hd"])
    del k
    x = torch.where(there, x, -math.inf)
    top = x.amax(3, keepdim=True).clamp_min(-3e38)                           # a row of no tokens has no largest score
    p = torch.exp(x - top)
    total = p.sum(3, keepdim=True)
    v = torch.where(there.transpose(2, 3), _gathered(s, "v"), 0.0)           # what lies behind the last token may be anything
    o = torch.matmul(p, v) / torch.where(total > 0, total, 1.0)
    s["out"].copy_(o.reshape(s["out"].shape))
    s["lse"].copy_((top + torch.log(total)).reshape(s["lse"].shape))
    return dict(out=s["out"], lse=s["lse"])


def _plain_append(s):
    t = torch.arange(s["k_new"].shape[0], device=DEV)
    if s["cu"] is None:
        row, back = t, torch.ones_like(t)
    else:
        row = torch.searchsorted(s["cu"][1:].contiguous(), t.int(), right=True)
        back = s["cu"][row + 1] - t                                          # tokens from this one to the row's end
    at = (s["lens"][row] - back).long()
    page = s["case"]["page"]
    p, slot = s["table"][row, at // page].long(), at % page

    def code(x, scale):
        if scale is None:
            return x
        return (x.float() / scale[0][:, None]).clamp(-FP8_MAX, FP8_MAX).to(torch.float8_e4m3fn).view(torch.uint8)

    s["k"][0][p, :, slot] = code(s["k_new"], s["k_scale"])
    s["v"][0][p, :, :, slot] = code(s["v_new"], s["v_scale"])
    return _pools(s)


def _plain_select(s, table, lens, src, table_out, lens_out):
    """Row r becomes the sequence src[r]: whole pages are shared, a part-filled last page stays with the first of its users and is
    copied for the others, sequences that nobody takes give their pages back."""
    page, width, n_in, n_out = s["case"]["page"], table.shape[1], table.shape[0], src.shape[0]
    src, rows, col = src.long(), torch.arange(n_out, device=DEV), torch.arange(width, device=DEV)
    n = lens[src]
    users = torch.zeros(n_in, dtype=torch.int32, device=DEV).scatter_add_(0, src, torch.ones_like(n))
    first = torch.full((n_in,), n_out, dtype=torch.int64, device=DEV).scatter_reduce_(0, src, rows, "amin")
    copied = (n % page > 0) & (first[src] != rows)
    free = torch.nonzero(s["refs"] == 0).flatten()
    new = free[(copied.cumsum(0) - 1).clamp_min(0)]
    # reference counts: a whole page counts its users, a part-filled one has one user, or none
    whole = col < (lens // page)[:, None]
    used = col < ((lens + page - 1) // page)[:, None]
    change = torch.where(whole, users[:, None], users[:, None].clamp_max(1)) - 1
    s["refs"].scatter_add_(0, table.clamp_min(0).long().flatten(), torch.where(used, change, 0).flatten())
    table_out.copy_(torch.where(col < ((n + page - 1) // page)[:, None], table[src], -1))
    r = torch.nonzero(copied).flatten()
    last = (n[r] // page).long()
    old = table_out[r, last].long()
    table_out[r, last] = new[r].int()
    s["refs"][new[r]] = 1
    s["k"][:, new[r]] = s["k"][:, old]
    s["v"][:, new[r]] = s["v"][:, old]
    lens_out.copy_(n)


def _plain_pages(s):
    page = s["case"]["page"]
    s["refs"].copy_(s["refs0"])
    if s["case"]["what"] == "compact":
        s["table"].copy_(s["table0"])
        live = s["refs"] > 0
        n = int(live.sum())
        holes = torch.nonzero(~live[:n]).flatten()
        moved = torch.nonzero(live[n:]).flatten() + n
        s["k"][:, holes] = s["k"][:, moved]
        s["v"][:, holes] = s["v"][:, moved]
        goes = torch.arange(live.shape[0], dtype=torch.int32, device=DEV)
        goes[moved] = holes.int()
        s["table"].copy_(torch.where(s["table"] >= 0, goes[s["table"].clamp_min(0).long()], -1))
        s["refs"][holes] = s["refs"][moved]
        s["refs"][moved] = 0
        return dict(table=s["table"], refs=s["refs"], **_pools(s))
    _plain_select(s, s["table"], s["lens"], s["expand"], s["table_many"], s["lens_many"])
    have, want = (s["lens_many"] + page - 1) // page, (s["lens_many"] + s["ones"] + page - 1) // page
    free = torch.nonzero(s["refs"] == 0).flatten()
    before = (want - have).cumsum(0) - (want - have)
    col = torch.arange(s["table_many"].shape[1], device=DEV)
    fresh = (col >= have[:, None]) & (col < want[:, None])
    s["table_many"].copy_(torch.where(fresh, free[(before[:, None] + col - have[:, None]).clamp(0, free.shape[0] - 1)].int(), s["table_many"]))
    s["refs"][s["table_many"][fresh].long()] = 1
    s["lens_grown"].copy_(s["lens_many"] + s["ones"])
    _plain_select(s, s["table_many"], s["lens_grown"], s["prune"], s["table_few"], s["lens_few"])
    return dict(many=s["table_many"], lens_many=s["lens_grown"], few=s["table_few"], lens_few=s["lens_few"], refs=s["refs"], **_pools(s))


def _plain_adjusted(s):
    z = s["logits"].float()
    R, V = z.shape
    if s["tokens"] is not None:
        at = torch.arange(s["tokens"].shape[1], device=DEV)
        told = at < s["n_tokens"][:, None]
        made = told & (at >= s["n_prompt"][:, None])
        ids = s["tokens"].long()
        count = torch.zeros(R, V, device=DEV).scatter_add_(1, ids, made.float())
        seen = torch.zeros(R, V, device=DEV).scatter_add_(1, ids, told.float()) > 0
        rep = s["repetition"][:, None]
        z = torch.where(seen, torch.where(z > 0, z / rep, z * rep), z)
        z = z - s["frequency"][:, None] * count
        z = torch.where(count > 0, z - s["presence"][:, None], z)
    if s["bias_ids"] is not None:
        n = s["bias_ids"].shape[0] - 1
        row = torch.searchsorted(s["bias_offsets"][1:].contiguous(), torch.arange(n, device=DEV, dtype=torch.int32), right=True)
        z = z.clone() if z is s["logits"] else z
        z[row, s["bias_ids"][:n].long()] += s["bias_values"][:n]
    if s["allow"] is not None:
        v = torch.arange(V, device=DEV)
        bits = (s["allow"][:, v // 32] >> (v % 32)) & 1 != 0                 # [masks, V]
        free = s["allow_row"] < 0
        z = torch.where(bits[s["allow_row"].clamp_min(0).long()] | free[:, None], z, -math.inf)
    return z


def _plain_adjust(s):
    s["out"].copy_(_plain_adjusted(s))
    return s["out"]


def _philox_round(state, r):
    """One round of Philox-4x32 on 64-bit integers that hold 32-bit words."""
    a, b, c, d, k0, k1 = state
    low = 0xFFFFFFFF
    p, q = 0xD2511F53 * a, 0xCD9E8D57 * c                                    # wrap modulo 2^64: the bits are the product's
    return ((q >> 32) & low ^ b ^ k0, q & low, (p >> 32) & low ^ d ^ k1, p & low, (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low)


def _plain_words(ids, vocab, key, step):
    """[rows, vocab] random words: word v mod 4 of the block with counter (v div 4, step, id, 2), key (low, high)."""
    blocks = torch.arange(-(-vocab // 4), device=DEV)[None].expand(ids.shape[0], -1)
    zero = torch.zeros_like(blocks)
    start = (blocks, zero + step, zero + ids.long()[:, None], zero + 2, key & 0xFFFFFFFF, key >> 32)
    words = functools.reduce(_philox_round, range(10), start)[:4]
    return torch.stack(words, 2).flatten(1)[:, :vocab]


def _plain_sample(s):
    z = _plain_adjusted(s)
    greedy = (s["temperature"] == 0)[:, None]
    y = z * (1.0 / torch.where(greedy, 1.0, s["temperature"][:, None]))
    w = ((_plain_words(s["ids"], z.shape[1], s["key"], s["step"]).float() + 0.5) * 2.0 ** -32).clamp_max(1 - 2.0 ** -24)
    score = torch.where(greedy, z, y - torch.log(-torch.log1p(-w)))
    best = score.amax(1, keepdim=True)
    v = torch.arange(z.shape[1], device=DEV)
    token = torch.where((score == best) & (best > -math.inf), v, z.shape[1]).amin(1)      # the lowest of equal ones
    none = token == z.shape[1]
    top = y.amax(1).clamp_min(-3e38)
    total = torch.exp(y - top[:, None]).sum(1)
    chosen = y.gather(1, token.clamp_max(z.shape[1] - 1)[:, None])[:, 0]
    s["token"].copy_(torch.where(none, -1, token))
    s["logp"].copy_(torch.where(none, -math.inf, chosen - top - torch.log(total)))
    return dict(token=s["token"], logp=s["logp"])


_own = dict(attend=_own_attend, append=_own_append, pages=_own_pages, adjust=_own_adjust, sample=_own_sample)
_plain = dict(attend=_plain_attend, append=_plain_append, pages=_plain_pages, adjust=_plain_adjust, sample=_plain_sample)


# ---------------------------------------------------------------- the definition in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    if case["work"] == "attend":
        out = torch.zeros(s["out"].shape, dtype=torch.float64, device=DEV)
        lse = torch.full(s["lse"].shape, -math.inf, dtype=torch.float64, device=DEV)
        group = case["heads"] // case["kv_heads"]
        for r, n in enumerate(_lengths(case["rows"], case["lo"], case["hi"])):
            row = s["table"][r, :_pages(n, case["page"])].long()
            k, v = _exact_values(s, "k", row), _exact_values(s, "v", row)
            k = k.permute(1, 0, 2, 3).reshape(case["kv_heads"], -1, case["hd"])[:, :n]
            v = v.permute(1, 0, 3, 2).reshape(case["kv_heads"], -1, case["hd"])[:, :n]
            for h in range(case["kv_heads"]):
                x = s["q"][r, h * group:(h + 1) * group].double() @ k[h].T / math.sqrt(case["hd"])
                lse[r, h * group:(h + 1) * group] = torch.logsumexp(x, 1)
                out[r, h * group:(h + 1) * group] = torch.softmax(x, 1) @ v[h]
        return dict(out=out, lse=lse)
    if case["work"] == "append":
        k, v = s["k"], s["v"]
        if s["k_scale"] is not None:
            k, v = k.view(torch.float8_e4m3fn), v.view(torch.float8_e4m3fn)
        k, v, t, page = k.double(), v.double(), 0, case["page"]
        x, y = s["k_new"].double(), s["v_new"].double()
        if s["k_scale"] is not None:                                         # before it is rounded
            x = (x / s["k_scale"][0].double()[:, None]).clamp(-FP8_MAX, FP8_MAX)
            y = (y / s["v_scale"][0].double()[:, None]).clamp(-FP8_MAX, FP8_MAX)
        table = s["table"].tolist()
        for r, n in enumerate(_lengths(case["rows"], case["lo"], case["hi"])):
            new = min(n, case["new"] or n)
            at = n - new
            while at < n:                                                    # what goes into one page
                m = min(page - at % page, n - at)
                p, lo = table[r][at // page], at % page
                k[0, p, :, lo:lo + m] = x[t:t + m].transpose(0, 1)
                v[0, p, :, :, lo:lo + m] = y[t:t + m].permute(1, 2, 0)
                at, t = at + m, t + m
        return dict(k=k, v=v)
    if case["work"] == "pages":
        return _exact_pages(case, s)
    return _exact_logits(case, s)


def _exact_values(s, name, pages):
    if s["k_scale"] is None:
        return s[name][0, pages].double()
    return s[name][0, pages].view(torch.float8_e4m3fn).double() * s[name + "_scale"][0].double()[:, None, None]


def _exact_pages(case, s):
    page, k, v = case["page"], s["k"].double(), s["v"].double()
    refs, table = s["refs0"].tolist(), (s["table0"] if case["what"] == "compact" else s["table"]).tolist()
    lens, width = s["lens"].tolist(), len(table[0])
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    padded = lambda rows: ints([row + [-1] * (width - len(row)) for row in rows])  # noqa: E731
    rows = [row[:_pages(n, page)] for row, n in zip(table, lens)]

    def move(old, new):
        k[:, new], v[:, new] = k[:, old], v[:, old]

    if case["what"] == "compact":
        n = sum(c > 0 for c in refs)
        goes = dict(zip([p for p in range(n, len(refs)) if refs[p]], [p for p in range(n) if not refs[p]]))
        for old, hole in goes.items():
            move(old, hole)
            refs[hole], refs[old] = refs[old], 0
        return dict(table=padded([[goes.get(p, p) for p in row] for row in rows]), refs=ints(refs), k=k, v=v)

    def select(rows, lens, src):
        got, owner, free = [], set(), [p for p, c in enumerate(refs) if not c]
        for r in src:
            row = list(rows[r])
            if r in owner:
                for p in row[:lens[r] // page]:
                    refs[p] += 1
                if lens[r] % page:
                    new = free.pop(0)
                    move(row[-1], new)
                    refs[new], row[-1] = 1, new
            owner.add(r)
            got.append(row)
        for r, row in enumerate(rows):
            if r not in owner:
                for p in row:
                    refs[p] -= 1
        return got, [lens[r] for r in src]

    rows, lens = select(rows, lens, s["expand"].tolist())
    for row, n in zip(rows, lens):
        if n % page == 0:
            row.append(refs.index(0))
            refs[row[-1]] = 1
    lens = [n + 1 for n in lens]
    many, lens_many = padded(rows), ints(lens)
    rows, lens = select(rows, lens, s["prune"].tolist())
    return dict(many=many, lens_many=lens_many, few=padded(rows), lens_few=ints(lens), refs=ints(refs), k=k, v=v)


def _exact_logits(case, s):
    R, V = case["rows"], case["vocab"]
    out = torch.empty(R, V, dtype=torch.float64, device=DEV) if case["work"] == "adjust" else None
    tokens, logps = [], []
    v = torch.arange(V, device=DEV)
    for r in range(R):
        z = s["logits"][r].double()
        if s["tokens"] is not None:
            n, m = int(s["n_tokens"][r]), int(s["n_prompt"][r])
            ids = s["tokens"][r].long()
            count = torch.bincount(ids[m:n], minlength=V)
            seen = torch.bincount(ids[:n], minlength=V) > 0
            rep = s["repetition"][r].double()
            z[seen] = torch.where(z[seen] > 0, z[seen] / rep, z[seen] * rep)
            z -= s["frequency"][r].double() * count + s["presence"][r].double() * (count > 0)
        if s["bias_ids"] is not None:
            a, b = int(s["bias_offsets"][r]), int(s["bias_offsets"][r + 1])
            z[s["bias_ids"][a:b].long()] += s["bias_values"][a:b].double()
        if s["allow"] is not None and int(s["allow_row"][r]) >= 0:
            words = s["allow"][int(s["allow_row"][r])].long() & 0xFFFFFFFF
            z[((words[v >> 5] >> (v & 31)) & 1) == 0] = -math.inf
        if out is not None:
            out[r] = z
            continue
        t = float(s["temperature"][r])
        y = z / (t or 1.0)
        if t:
            w = (_exact_words(v // 4, s["step"], int(s["ids"][r]), s["key"]).gather(0, (v % 4)[None])[0].double() + 0.5) / 2 ** 32
            score = y - torch.log(-torch.log1p(-w.clamp_max(1 - 2.0 ** -24)))
        else:
            score = z
        best = int(torch.nonzero(score == score.max())[0])
        none = not math.isfinite(float(score[best]))
        tokens.append(-1 if none else best)
        logps.append(-math.inf if none else float(y[best] - torch.logsumexp(y, 0)))
    if out is not None:
        return out
    return dict(token=torch.tensor(tokens, dtype=torch.int32), logp=torch.tensor(logps, dtype=torch.float64))


def _exact_words(block, step, row, key):
    """[4, n] words of Philox-4x32-10, its products taken in halves of 16 bits."""
    mask, half = (1 << 32) - 1, (1 << 16) - 1

    def product(m, x):
        lo, hi = (m & half) * x, (m >> 16) * x
        total = lo + ((hi & half) << 16)
        return (hi >> 16) + (total >> 32) & mask, total & mask

    c = [block.long(), torch.full_like(block, step), torch.full_like(block, row), torch.full_like(block, 2)]
    key = [key & mask, key >> 32]
    for i in range(10):
        h0, l0 = product(0xD2511F53, c[0])
        h1, l1 = product(0xCD9E8D57, c[2])
        c = [h1 ^ c[1] ^ key[0], l1, h0 ^ c[3] ^ key[1], l0]
        key = [(key[0] + 0x9E3779B9) & mask, (key[1] + 0xBB67AE85) & mask]
    return torch.stack(c)
