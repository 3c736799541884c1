"""What a token policy learns from, as its users call it: for timing, and for comparing the kernels with their plain forms.

Four kinds of work over rows of logits or of log-probs:
  score      log-probs of given tokens, entropies and the most likely alternatives (pg_token_logprobs)
  policy     the same without alternatives, and the gradient of the logits (pg_token_logprobs, pg_token_logprobs_backward)
  distill    divergence from a teacher's most likely tokens, and the gradient of the logits (pg_distill_loss, pg_distill_backward)
  surrogate  the clipped objective of sequences and the gradient of their tokens' log-probs (pg_token_surrogate)

Which rows are padding, how long sequences and lists are and which rows a mask is for follow from the case; values come from the seed.
"""
import math

import torch

own = False
DEV = "cuda:0"


def listed():
    return [
        # ---- log-probs ----
        # the token that was just drawn for one request, with 20 alternatives: latency
        dict(name="score_one", work="score", rows=1, vocab=32001, dtype="f32", n_top=20, masks=0, pad=0, warm=1),
        # a group of 48 over a codebook under a grammar, five alternatives
        dict(name="score_group", work="score", rows=48, vocab=16384, dtype="f32", n_top=5, masks=4, pad=0, warm=1),
        # all tokens of a long prompt over an odd vocabulary, log-probs and entropies alone
        dict(name="score_prompt", work="score", rows=4096, vocab=65537, dtype="bf16", n_top=0, masks=0, pad=0, warm=0),
        # a teacher's 64 most likely tokens for a batch of sequences
        dict(name="score_teacher", work="score", rows=1178, vocab=131073, dtype="bf16", n_top=64, masks=0, pad=0, warm=0),
        # ---- log-probs and their gradient ----
        # one step of a small group
        dict(name="policy_group", work="policy", rows=48, vocab=16384, dtype="f32", masks=0, pad=0, warm=1, entropy=1),
        # sequences padded to one length, grammar masks, odd vocabulary
        dict(name="policy_masked", work="policy", rows=1178, vocab=65537, dtype="bf16", masks=16, pad=8, warm=1, entropy=1),
        # a micro-batch over a large vocabulary
        dict(name="policy_batch", work="policy", rows=4096, vocab=131072, dtype="bf16", masks=0, pad=0, warm=0, entropy=1),
        # ---- distillation ----
        # a few rows, short lists, the teacher's probabilities renormalised over them
        dict(name="distill_group", work="distill", rows=48, vocab=32001, dtype="f32", k=20, tail=0, masks=0, warm=0),
        # a micro-batch, what the teacher leaves out as one more outcome
        dict(name="distill_batch", work="distill", rows=2048, vocab=131073, dtype="bf16", k=64, tail=1, masks=0, warm=1),
        # ---- surrogate ----
        # a group of 48 sequences
        dict(name="surrogate_group", work="surrogate", seqs=48, lo=1, hi=1178, ref=1, weighted=0),
        # eight groups of 48 long sequences
        dict(name="surrogate_batch", work="surrogate", seqs=384, lo=1, hi=16384, ref=1, weighted=1),
        # few very long ones
        dict(name="surrogate_long", work="surrogate", seqs=3, lo=65537, hi=131071, ref=0, weighted=0),
    ]


def draw(rng):
    def log_int(lo, hi):
        return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))

    work = rng.choice(["score", "policy", "policy", "distill", "distill", "surrogate"])
    if work == "surrogate":
        seqs = log_int(1, 512)
        hi = log_int(1, min(131071, 6_000_000 // seqs))
        return dict(work=work, seqs=seqs, lo=log_int(1, hi), hi=hi, ref=rng.choice([0, 1]), weighted=rng.choice([0, 1]))
    rows, vocab = log_int(1, 4096), log_int(200, 131073)
    while rows * vocab > 2 ** 28:
        rows = rows * 3 // 4
    c = dict(work=work, rows=rows, vocab=vocab, dtype=rng.choice(["f32", "bf16"]), masks=rng.choice([0, 0, 1, 16]), warm=rng.choice([0, 1]))
    if work == "score":
        if rows * vocab > 2 ** 27:
            c["rows"] = max(1, 2 ** 27 // vocab)
        return dict(c, n_top=rng.choice([0, 1, 5, 20, 64]), pad=rng.choice([0, 0, 8]))
    if work == "policy":
        return dict(c, pad=rng.choice([0, 0, 3, 8]), entropy=rng.choice([0, 1, 1]))
    return dict(c, k=log_int(1, 128), tail=rng.choice([0, 1]))


# ---------------------------------------------------------------- what a user's program has in hand

def _lengths(rows, lo, hi):
    """Lengths between lo and hi, spread evenly in a scattered order; the first has the longest."""
    return [hi if r == 0 else lo + int(((r * 0.6180339887498949) % 1.0) * (hi - lo + 1)) for r in range(rows)]


def _padding(case):
    """Rows without a token of their own."""
    return [bool(case.get("pad")) and r % case["pad"] == case["pad"] - 1 for r in range(case["rows"])]


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    normal = lambda *shape: torch.randn(*shape, device=DEV, generator=gen)  # noqa: E731
    s = dict(case=case)
    if case["work"] == "surrogate":
        lengths = _lengths(case["seqs"], case["lo"], case["hi"])
        n = sum(lengths)
        s["cu"] = ints([0] + torch.tensor(lengths).cumsum(0).tolist())
        s["logp"] = -normal(n).abs() * 2
        s["logp_old"] = s["logp"] + normal(n) * 0.15
        s["logp_ref"] = s["logp"] + normal(n) * 0.3 if case["ref"] else None
        s["adv"] = normal(case["seqs"])
        s["weight"] = torch.full((case["seqs"],), 1 / n, device=DEV) if case["weighted"] else None
        s.update(clip_low=0.2, clip_high=0.28, kl_coef=0.04)
        for name in ("objective", "kl"):
            s[name] = torch.empty(case["seqs"], device=DEV)
        s["clipped"] = torch.empty(case["seqs"], dtype=torch.int32, device=DEV)
        s["g_logp"] = torch.empty(n, device=DEV)
        return s
    R, V = case["rows"], case["vocab"]
    kind = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
    s["logits"] = torch.empty(R, V, dtype=kind, device=DEV)
    part = max(1, 2 ** 26 // V)
    for r in range(0, R, part):
        s["logits"][r:r + part] = normal(min(part, R - r), V) * 3
    s["allow"] = s["allow_row"] = s["temperature"] = None
    if case["warm"]:
        s["temperature"] = 0.7 + 0.6 * torch.rand(R, device=DEV, generator=gen)
    if case["masks"]:
        m, words = case["masks"], -(-V // 32)
        a = torch.randint(-2 ** 31, 2 ** 31, (m, words), device=DEV, generator=gen).to(torch.int32)
        # of more than one mask the last allows nothing; a row in four has no mask
        if m > 1:
            a[m - 1] = 0
        s["allow"] = a
        s["allow_row"] = ints([-1 if r % 4 == 3 else m - 1 if r == 5 else r % max(1, m - 1) for r in range(R)])
    rows = torch.arange(R, device=DEV)
    if case["work"] == "distill":
        # the teacher agrees with the student in part; its lists are of different lengths, and one is empty
        k = min(case["k"], V)
        s["teacher_ids"] = torch.empty(R, k, dtype=torch.int32, device=DEV)
        s["teacher_logp"] = torch.empty(R, k, device=DEV)
        for r in range(0, R, part):
            t = s["logits"][r:r + part].float() * 0.8 + normal(min(part, R - r), V) * 1.8
            if s["allow"] is not None:
                t = torch.where(_allowed(s, r, r + part), t, -20.0)
            top, ids = t.topk(k)
            s["teacher_ids"][r:r + part] = ids
            s["teacher_logp"][r:r + part] = top - t.logsumexp(1, keepdim=True)
        n = [0 if r == 7 else k - (r % 5) * k // 16 for r in range(R)]
        gone = torch.arange(k, device=DEV)[None, :] >= torch.tensor(n, device=DEV)[:, None]
        s["teacher_ids"][gone] = -1
        s["teacher_logp"][gone] = -math.inf
        s["g_loss"] = torch.rand(R, device=DEV, generator=gen) / R
        s["loss"] = torch.empty(R, device=DEV)
    else:
        # a likely token: the best allowed one of sixteen
        some = torch.randint(0, V, (R, 16), device=DEV, generator=gen)
        value = s["logits"].gather(1, some).float()
        if s["allow"] is not None:
            value = torch.where(_bits(s, rows[:, None], some), value, -math.inf)
        target = some.gather(1, value.argmax(1, keepdim=True))[:, 0]
        s["target"] = torch.where(torch.tensor(_padding(case), device=DEV), -1, target).to(torch.int32)
        s["logp"], s["entropy"] = torch.empty(R, device=DEV), torch.empty(R, device=DEV)
        if case.get("n_top"):
            s["top_ids"] = torch.empty(R, case["n_top"], dtype=torch.int32, device=DEV)
            s["top_logp"] = torch.empty(R, case["n_top"], device=DEV)
        s["g_logp"] = normal(R) / R
        s["g_entropy"] = torch.full((R,), 0.01 / R, device=DEV) if case.get("entropy") else None
    if case["work"] != "score":
        s["d_logits"] = torch.empty_like(s["logits"])
    return s


def _bits(s, row, token):
    """Whether the tokens are allowed in the rows."""
    mask = s["allow_row"].long()[row]
    word = s["allow"][mask.clamp_min(0), token >> 5]
    return (mask < 0) | ((word >> (token & 31)) & 1).bool()


def _allowed(s, lo, hi):
    R, V = s["logits"].shape
    hi = min(hi, R)
    return _bits(s, torch.arange(lo, hi, device=DEV)[:, None], torch.arange(V, device=DEV)[None, :])


def work(case):
    if case["work"] == "surrogate":
        n = sum(_lengths(case["seqs"], case["lo"], case["hi"]))
        return dict(bytes=n * (16 if case["ref"] else 12) + 24 * case["seqs"], flops=20 * n)
    elt = 4 if case["dtype"] == "f32" else 2
    live = case["rows"] - sum(_padding(case))
    masks = case["masks"] * (-(-case["vocab"] // 32)) * 4
    once = live * case["vocab"]
    if case["work"] == "score":
        return dict(bytes=once * elt + masks + case["rows"] * (12 + 8 * case["n_top"]), flops=6 * once)
    grad = case["rows"] * case["vocab"] * elt
    if case["work"] == "policy":
        return dict(bytes=once * elt + masks + grad + 16 * case["rows"], flops=14 * once)
    return dict(bytes=once * elt + masks + grad + case["rows"] * (8 * min(case["k"], case["vocab"]) + 8), flops=10 * once)


# ---------------------------------------------------------------- one pass

def run(s):
    return (_own if own else _plain)[s["case"]["work"]](s)


# ---- the framework's calls

def _descriptor(s):
    """The handle that a program keeps beside its logits, and the scratch of its calls."""
    from paper_2512_15347_amd import binding as pg
    if "descriptor" not in s:
        c = s["case"]
        s["descriptor"] = pg.Logits(s["logits"], allow=s["allow"], allow_row=s["allow_row"])
        need = pg.pg_distill_scratch_floats(c["rows"], c["vocab"]) if c["work"] == "distill" else \
            pg.pg_logprob_scratch_floats(c["rows"], c["vocab"], c.get("n_top", 0))
        s["scratch"] = torch.empty(need, device=DEV)
        s["stats"] = torch.empty(c["rows"], pg.PG_DISTILL_STATS if c["work"] == "distill" else pg.PG_LOGPROB_STATS, device=DEV)
    return pg, s["descriptor"]


def _own_score(s):
    pg, d = _descriptor(s)
    n = s["case"]["n_top"]
    top = dict(top_ids=s["top_ids"], top_logp=s["top_logp"]) if n else {}
    pg.pg_token_logprobs(d, s["target"], s["logp"], s["scratch"], temperature=s["temperature"], entropy=s["entropy"], **top)
    return dict(logp=s["logp"], entropy=s["entropy"], **top)


def _own_policy(s):
    pg, d = _descriptor(s)
    pg.pg_token_logprobs(d, s["target"], s["logp"], s["scratch"], temperature=s["temperature"], entropy=s["entropy"], stats=s["stats"])
    pg.pg_token_logprobs_backward(d, s["target"], s["stats"], s["d_logits"], g_logp=s["g_logp"], g_entropy=s["g_entropy"],
                                  temperature=s["temperature"])
    return dict(logp=s["logp"], entropy=s["entropy"], d_logits=s["d_logits"])


def _own_distill(s):
    pg, d = _descriptor(s)
    pg.pg_distill_loss(d, s["teacher_ids"], s["teacher_logp"], s["loss"], s["scratch"], tail=bool(s["case"]["tail"]),
                       temperature=s["temperature"], stats=s["stats"])
    pg.pg_distill_backward(d, s["teacher_ids"], s["teacher_logp"], s["stats"], s["g_loss"], s["d_logits"], temperature=s["temperature"])
    return dict(loss=s["loss"], d_logits=s["d_logits"])


def _own_surrogate(s):
    from paper_2512_15347_amd import binding as pg
    c = s["case"]
    if "scratch" not in s:
        s["scratch"] = torch.empty(pg.pg_surrogate_scratch_floats(c["seqs"], c["hi"]), device=DEV)
    pg.pg_token_surrogate(s["logp"], s["logp_old"], s["adv"], s["cu"], s["objective"], s["g_logp"], s["clip_low"], s["clip_high"], c["hi"],
                          s["scratch"], logp_ref=s["logp_ref"], kl_coef=s["kl_coef"], weight=s["weight"], kl=s["kl"], clipped=s["clipped"])
    return {k: s[k] for k in ("objective", "kl", "clipped", "g_logp") if k != "kl" or c["ref"]}


_own = dict(score=_own_score, policy=_own_policy, distill=_own_distill, surrogate=_own_surrogate)


# ---- the plain forms

def _scaled(s):
    """y in fp32, with -inf where a token is not allowed, and 1 / temperature."""
    z = s["logits"].float()
    if s["allow"] is not None:
        z = torch.where(_allowed(s, 0, z.shape[0]), z, -math.inf)
    inv = torch.ones(z.shape[0], device=DEV) if s["temperature"] is None else 1 / s["temperature"]
    return z * inv[:, None], inv


def _softmax_parts(y):
    """(y - largest, exp of it, ln of its sum): zeros and -inf where nothing is allowed."""
    top = y.amax(1, keepdim=True)
    shifted = y - torch.where(top == -math.inf, 0.0, top)
    e = torch.exp(shifted)
    return shifted, e, torch.log(e.sum(1, keepdim=True))


def _plain_forward(s, y):
    shifted, e, ln_sum = _softmax_parts(y)
    total = e.sum(1, keepdim=True)
    mean = torch.where(e > 0, e * shifted, 0.0).sum(1, keepdim=True) / torch.where(total > 0, total, 1.0)
    entropy = torch.where(total > 0, ln_sum - mean, 0.0)
    logq = torch.where(total > 0, shifted - ln_sum, -math.inf)
    target = s["target"].long()
    logp = logq.gather(1, target.clamp_min(0)[:, None])[:, 0]
    here = target >= 0
    return logq, torch.where(here, logp, 0.0), torch.where(here, entropy[:, 0], 0.0), here


def _plain_score(s):
    y, _ = _scaled(s)
    logq, logp, entropy, here = _plain_forward(s, y)
    out = dict(logp=logp, entropy=entropy)
    n = s["case"]["n_top"]
    if n:
        # equal logits in the order of their numbers: both in one integer, whose order is that of the logits
        bits = torch.where(y == -math.inf, -math.inf, s["logits"].float() + 0.0).view(torch.int32)
        V = y.shape[1]
        key = (torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long() << 32) | (V - 1 - torch.arange(V, device=DEV))[None, :]
        best = key.topk(min(n, V), sorted=True)[0]
        ids = V - 1 - (best & 0xFFFFFFFF)
        value = logq.gather(1, ids)
        none = (value == -math.inf) | ~here[:, None]
        out["top_ids"] = torch.full((y.shape[0], n), -1, dtype=torch.int32, device=DEV)
        out["top_logp"] = torch.full((y.shape[0], n), -math.inf, device=DEV)
        out["top_ids"][:, :ids.shape[1]] = torch.where(none, -1, ids).to(torch.int32)
        out["top_logp"][:, :ids.shape[1]] = torch.where(none, -math.inf, value)
    return out


def _plain_policy(s):
    y, inv = _scaled(s)
    logq, logp, entropy, here = _plain_forward(s, y)
    p = torch.exp(logq)
    g = torch.where(here, s["g_logp"], 0.0)[:, None]
    d = -g * p
    if s["g_entropy"] is not None:
        ge = torch.where(here, s["g_entropy"], 0.0)[:, None]
        d = d - torch.where(p > 0, ge * p * (logq + entropy[:, None]), 0.0)
    at = s["target"].long().clamp_min(0)[:, None]
    d.scatter_add_(1, at, torch.where(logq.gather(1, at) > -math.inf, g, 0.0))
    return dict(logp=logp, entropy=entropy, d_logits=(d * inv[:, None]).to(s["logits"].dtype))


def _plain_distill(s):
    y, inv = _scaled(s)
    ids, t = s["teacher_ids"].long(), s["teacher_logp"].double()
    there = ids >= 0
    row = there.any(1, keepdim=True) & (y > -math.inf).any(1, keepdim=True)      # of the others nothing is learnt
    at = ids.clamp_min(0)
    is_listed = torch.zeros(y.shape, dtype=torch.int8, device=DEV).scatter_add_(1, at, there.to(torch.int8)) > 0
    shifted, e, ln_sum = _softmax_parts(y)
    e_rest = torch.where(is_listed, 0.0, e)
    p_rest = (e_rest.sum(1, keepdim=True) / e.sum(1, keepdim=True)).double()
    q = torch.where(there, torch.exp(t), 0.0)
    if s["case"]["tail"]:
        q_rest = torch.where(p_rest > 0, (1 - q.sum(1, keepdim=True)).clamp_min(0), 0.0)
    else:
        q, q_rest = q / q.sum(1, keepdim=True), torch.zeros_like(p_rest)
    logp = (shifted.gather(1, at) - ln_sum).double()
    loss = torch.where(q > 0, q * (torch.log(q) - logp), 0.0).sum(1, keepdim=True)
    loss = loss + torch.where(q_rest > 0, q_rest * (torch.log(q_rest) - torch.log(p_rest)), 0.0)
    everything = q.sum(1, keepdim=True) + q_rest
    g = s["g_loss"][:, None] * inv[:, None]
    rest = torch.where(p_rest > 0, everything - q_rest / p_rest, 0.0).float()
    p = torch.exp(shifted - ln_sum)
    d = p * torch.where(is_listed, everything.float(), rest)
    d.scatter_add_(1, at, torch.where(there & (logp > -math.inf), -q, 0.0).float())
    d = torch.where(row, d * g, 0.0)
    return dict(loss=torch.where(row, loss, 0.0)[:, 0].float(), d_logits=d.to(s["logits"].dtype))


def _segments(x, cu):
    """Sums over the sequences."""
    ends = torch.cat([torch.zeros(1, dtype=x.dtype, device=DEV), x.cumsum(0)])
    cu = cu.long()
    return ends[cu[1:]] - ends[cu[:-1]]


def _plain_surrogate(s):
    cu = s["cu"].long()
    n = cu[1:] - cu[:-1]
    seq = torch.repeat_interleave(torch.arange(n.shape[0], device=DEV), n, output_size=s["logp"].shape[0])
    logp, a = s["logp"].double(), s["adv"].double()[seq]
    w = (1 / n.double() if s["weight"] is None else s["weight"].double())
    ratio = torch.exp(logp - s["logp_old"].double())
    lo, hi = 1 - s["clip_low"], 1 + s["clip_high"]
    cut = ((a > 0) & (ratio > hi)) | ((a < 0) & (ratio < lo))
    term = torch.minimum(ratio * a, ratio.clamp(lo, hi) * a)
    g = torch.where(cut, 0.0, ratio * a)
    out = {}
    if s["logp_ref"] is not None:
        x = s["logp_ref"].double() - logp
        k = torch.exp(x) - x - 1
        term, g = term - s["kl_coef"] * k, g + s["kl_coef"] * (torch.exp(x) - 1)
        out["kl"] = (_segments(k, cu) / n).float()
    return dict(objective=(_segments(term, cu) * w).float(), clipped=_segments(cut.int(), cu).int(), g_logp=(g * w[seq]).float(), **out)


_plain = dict(score=_plain_score, policy=_plain_policy, distill=_plain_distill, surrogate=_plain_surrogate)


# ---------------------------------------------------------------- the definitions in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    if case["work"] == "surrogate":
        cu = s["cu"].tolist()
        parts = dict(objective=[], kl=[], g_logp=[])
        for r in range(case["seqs"]):
            at = slice(cu[r], cu[r + 1])
            d, a = s["logp"][at].double() - s["logp_old"][at].double(), float(s["adv"][r])
            w = float(s["weight"][r]) if case["weighted"] else 1 / (cu[r + 1] - cu[r])
            inside = d <= math.log1p(s["clip_high"]) if a > 0 else d >= math.log1p(-s["clip_low"])
            bound = 1 + s["clip_high"] if a > 0 else 1 - s["clip_low"]
            value, slope = torch.where(inside, d.exp(), bound) * a, torch.where(inside, d.exp() * a, 0.0)
            if case["ref"]:
                x = s["logp_ref"][at].double() - s["logp"][at].double()
                value, slope = value - s["kl_coef"] * (x.expm1() - x), slope + s["kl_coef"] * x.expm1()
                parts["kl"].append((x.expm1() - x).mean())
            parts["objective"].append(value.sum() * w)
            parts["g_logp"].append(slope * w)
        out = dict(objective=torch.stack(parts["objective"]), g_logp=torch.cat(parts["g_logp"]), clipped=None)
        return dict(out, kl=torch.stack(parts["kl"])) if case["ref"] else out
    step = max(1, 2 ** 26 // case["vocab"])
    parts = [_exact_rows(s, r, min(r + step, case["rows"])) for r in range(0, case["rows"], step)]
    return {k: None if parts[0][k] is None else torch.cat([p[k] for p in parts]) for k in parts[0]}


def _exact_rows(s, lo, hi):
    case, rows = s["case"], torch.arange(hi - lo, device=DEV)
    t = torch.ones(hi - lo, dtype=torch.float64, device=DEV) if s["temperature"] is None else s["temperature"][lo:hi].double()
    y = s["logits"][lo:hi].double() / t[:, None]
    open_ = torch.ones_like(y, dtype=torch.bool) if s["allow"] is None else _allowed(s, lo, hi)
    y = y.masked_fill(~open_, -math.inf)
    lse = torch.logsumexp(y, 1)
    some = open_.any(1)                                  # rows that allow a token
    ln = (y - lse[:, None]).masked_fill(~open_, -math.inf)
    p = ln.exp()
    plog = torch.nan_to_num(p * ln, nan=0.0)
    if case["work"] == "distill":
        ids, g = s["teacher_ids"][lo:hi].long(), s["g_loss"][lo:hi].double() / t
        q = torch.zeros(hi - lo, y.shape[1] + 1, dtype=torch.float64, device=DEV)      # the last column takes what is not there
        at = torch.where(ids >= 0, ids, y.shape[1])
        q.scatter_(1, at, s["teacher_logp"][lo:hi].double().exp())
        is_in = torch.zeros_like(q, dtype=torch.bool).scatter_(1, at, torch.ones_like(at, dtype=torch.bool))[:, :-1]
        q = q[:, :-1]
        learns = is_in.any(1) & some
        p_rest = p.masked_fill(is_in, 0.0).sum(1)
        q_rest = torch.zeros_like(p_rest)
        if case["tail"]:
            q_rest = torch.where((open_ & ~is_in).any(1), (1 - q.sum(1)).clamp_min(0), 0.0)
        else:
            q = q / q.sum(1, keepdim=True)
        loss = (torch.special.xlogy(q, q) - torch.where(q > 0, q * ln, 0.0)).sum(1) + torch.special.xlogy(q_rest, q_rest / p_rest)
        d = p * (q.sum(1) + q_rest)[:, None] - torch.where(open_, q, 0.0)
        d = d - torch.where(is_in, 0.0, p * (q_rest / p_rest.clamp_min(1e-300))[:, None])
        return dict(loss=torch.where(learns, loss, 0.0), d_logits=torch.where(learns[:, None], d * g[:, None], 0.0))
    target = s["target"][lo:hi].long()
    real = target >= 0
    at = target.clamp_min(0)
    entropy = torch.where(real & some, -plog.sum(1), 0.0)
    out = dict(logp=torch.where(real, torch.where(some, ln[rows, at], -math.inf), 0.0), entropy=entropy)
    if case["work"] == "score":
        n = case["n_top"]
        if n:
            value = torch.full((hi - lo, n), -math.inf, dtype=torch.float64, device=DEV)
            m = min(n, y.shape[1])
            value[:, :m] = ln.topk(m)[0]
            out.update(top_ids=None, top_logp=value.masked_fill(~(real & some)[:, None], -math.inf))
        return out
    g = s["g_logp"][lo:hi].double() * real
    d = -g[:, None] * p
    d[rows, at] += torch.where(open_[rows, at], g, 0.0)
    if s["g_entropy"] is not None:
        d = d - (s["g_entropy"][lo:hi].double() * real)[:, None] * (plog + p * entropy[:, None])
    return dict(out, d_logits=torch.where(some[:, None], d / t[:, None], 0.0))
