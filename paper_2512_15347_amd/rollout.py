"""Expand and prune for a policy that emits tokens: the group funnel of the sampling loop, with sequences in place of latents.

Each prompt is expanded to a group of members that share its pages, members draw their tokens from the policy's softmax, and at the
checkpoints Optimal Variance Filtering keeps the subset of each group whose proxy rewards vary most; the others' pages go back
to the pool.  Log-probs by original id and group-relative advantages come out, as from the denoising loop.  What the policy learns from them
follows: log-probs of the drawn tokens under other weights, the clipped objective with its gradient, or a teacher's distribution.

    python -m paper_2512_15347_amd.rollout

runs a small decoder with seeded random weights.  PyTorch is used for embeddings, norms, activations and index arithmetic around the
library's calls; nothing is copied to the host between the prompt and the advantages.
"""
import math

import numpy as np
import torch

from . import binding as pg
from .workloads import MASTER_SEED

# a decoder of the size of the reduced networks in workloads.py
SMALL = dict(D=256, blocks=2, heads=4, kv_heads=2, vocab=1000, page=16, max_len=256)


def make_weights(cfg, seed=MASTER_SEED, device="cuda:0"):
    """Seeded weights, N(0, 1 / inputs), matrices [out, in] in bf16."""
    g = torch.Generator().manual_seed(seed)

    def matrix(rows, cols):
        return (torch.randn(rows, cols, generator=g) / math.sqrt(cols)).to(torch.bfloat16).to(device)

    D, hd = cfg["D"], cfg["D"] // cfg["heads"]
    block = lambda: dict(qkv=matrix(D + 2 * cfg["kv_heads"] * hd, D), o=matrix(D, D), fc1=matrix(4 * D, D), fc2=matrix(D, 4 * D))  # noqa: E731
    return dict(embed=matrix(cfg["vocab"], D).float() * math.sqrt(D), position=matrix(cfg["max_len"], D).float(),
                blocks=[block() for _ in range(cfg["blocks"])], head=matrix(cfg["vocab"], D) * 4)


def _linear(x, w):
    """x w^T in fp32 from bf16 operands."""
    out = torch.empty(x.shape[0], w.shape[0], device=x.device)
    pg.pg_gemm_bf16(x, x.shape[1], w, w.shape[1], None, out, w.shape[0], x.shape[0], w.shape[0], w.shape[1])
    return out


def _norm(x):
    return (x * torch.rsqrt(x.square().mean(1, keepdim=True) + 1e-6)).to(torch.bfloat16)


class Decoder:
    """The policy: embedding, blocks of attention over the paged cache and an MLP, logits."""

    def __init__(self, cfg, weights, rows, device="cuda:0"):
        self.cfg, self.w, self.hd = cfg, weights, cfg["D"] // cfg["heads"]
        self.width = -(-cfg["max_len"] // cfg["page"])
        # every member may hold a row of its own, and a fork takes its copies before the old rows are given back
        self.cache = pg.Cache.create(cfg["blocks"], 2 * rows * self.width, cfg["kv_heads"], cfg["page"], self.hd, self.width, device=device)
        self.workspace = None

    def forward(self, *tokens, **more):
        """Logits that follow `tokens`; arguments as of hidden()."""
        return _linear(self.hidden(*tokens, **more), self.w["head"])

    def hidden(self, tokens, positions, table, lens, kv_len, row_of=None, cu=None):
        """What the logits are made of, for `tokens` (the last cu[r] .. cu[r+1]-1 of row r, or one a row); token i attends to kv_len[i] tokens of
        its row."""
        c, hd, n = self.cfg, self.hd, tokens.shape[0]
        need = pg.pg_paged_attention_workspace(self.cache, n, c["heads"], c["max_len"])
        if self.workspace is None or self.workspace.numel() < need:
            self.workspace = torch.empty(max(need, 16), dtype=torch.uint8, device=tokens.device)
        x = self.w["embed"][tokens.long()] + self.w["position"][positions.long()]
        for layer, w in enumerate(self.w["blocks"]):
            qkv = _linear(_norm(x), w["qkv"]).to(torch.bfloat16).view(n, -1, hd)
            q, k, v = qkv.split([c["heads"], c["kv_heads"], c["kv_heads"]], 1)
            pg.pg_cache_append(self.cache, layer, k, v, table, lens, cu=cu)
            out = torch.empty(n, c["heads"], hd, dtype=torch.bfloat16, device=x.device)
            pg.pg_paged_attention(self.cache, layer, q, table, kv_len, out, c["max_len"], self.workspace, row_of=row_of)
            x = x + _linear(out.view(n, -1), w["o"])
            x = x + _linear(torch.nn.functional.gelu(_linear(_norm(x), w["fc1"]), approximate="tanh").to(torch.bfloat16), w["fc2"])
        return _norm(x)


def sample_groups(decoder, prompts, members, steps, schedule, seed, token_reward, temperature=1.0, penalties=None, allow=None, adv_eps=1e-6):
    """prompts: list of token lists; schedule: [(step, k)], after which step k members of every group are kept (counts that fall with the
    steps, in any order).

    token_reward: fp32 [vocab]; a sequence's proxy reward is the mean over its drawn tokens.  penalties: (repetition, frequency, presence).
    allow: int32 [1, words] mask of tokens that may be drawn.  Returns survivors' ids, tokens, rewards and advantages, logp [steps,
    groups * members] by original id (NaN where pruned), and the penalties.  Raises PgError if pages ran out, a member had nothing to draw from or
    a reward at a checkpoint was no number."""
    dev, c, P = token_reward.device, decoder.cfg, len(prompts)
    if min(len(p) for p in prompts) < 1 or max(len(p) for p in prompts) + steps > c["max_len"] + 1:
        raise ValueError("prompts of at least one token that leave room for the steps are needed")
    if token_reward.shape != (c["vocab"],) or not all(0 <= t < c["vocab"] for p in prompts for t in p):
        raise ValueError("tokens of the prompts outside the vocabulary, or rewards for another one")
    keep, counts = dict(schedule), [members] + [k for _, k in sorted(schedule)]
    if len(keep) < len(schedule) or any(not 0 < k <= n for n, k in zip(counts, counts[1:])) or members > 64:
        raise ValueError("schedule: at most one count a step, falling from the group's members, at most 64")
    ints = lambda a: torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(dev)  # noqa: E731
    cache, width, M = decoder.cache, decoder.width, P * members
    pg.pg_cache_clear(cache)
    scratch = torch.empty(pg.pg_cache_scratch_ints(cache, M), dtype=torch.int32, device=dev)
    # the prompts, all of their tokens at once: token i of a row attends to its first i + 1 tokens
    sizes = [len(p) for p in prompts]
    table, lens = torch.full((P, width), -1, dtype=torch.int32, device=dev), torch.zeros(P, dtype=torch.int32, device=dev)
    pg.pg_cache_reserve(cache, table, lens, ints(sizes), lens)
    at = np.concatenate([np.arange(n) for n in sizes])
    decoder_in = ints(np.concatenate(prompts)), ints(at), table, lens, ints(at + 1)
    logits = decoder.forward(*decoder_in, row_of=ints(np.repeat(np.arange(P), sizes)), cu=ints(np.cumsum([0] + sizes)))
    logits = logits[torch.from_numpy(np.cumsum(sizes) - 1).to(dev)]
    # expansion: every member's row is its prompt's; whole pages are shared
    src = ints(np.repeat(np.arange(P), members))
    ids = torch.arange(M, dtype=torch.int32, device=dev)
    history = torch.zeros(P, max(sizes) + steps, dtype=torch.int32, device=dev)
    for g, p in enumerate(prompts):
        history[g, :len(p)] = ints(p)
    n_prompt = ints(sizes)

    def take(src, table, lens):
        new, new_lens = torch.empty(src.shape[0], width, dtype=torch.int32, device=dev), torch.empty(src.shape[0], dtype=torch.int32, device=dev)
        pg.pg_cache_select(cache, table, lens, src, new, new_lens, scratch)
        return new, new_lens

    table, lens = take(src, table, lens)
    rows = src.long()
    logits, history, n_prompt = logits[rows].contiguous(), history[rows].contiguous(), n_prompt[rows].contiguous()
    offsets = ints(np.arange(P + 1) * members)
    logp, score = torch.full((steps, M), math.nan, device=dev), torch.zeros(M, device=dev)
    undrawn = torch.zeros((), dtype=torch.bool, device=dev)             # some member had nothing to draw from
    status = torch.zeros(4, dtype=torch.int32, device=dev)              # of all selections
    for step in range(steps):
        n = ids.shape[0]
        more = {}
        if penalties is not None:
            fill = lambda v: torch.full((n,), float(v), device=dev)  # noqa: E731
            more = dict(tokens=history, n_prompt=n_prompt, n_tokens=n_prompt + step, repetition=fill(penalties[0]), frequency=fill(penalties[1]),
                        presence=fill(penalties[2]))
        if allow is not None:
            more.update(allow=allow, allow_row=torch.zeros(n, dtype=torch.int32, device=dev))
        desc = pg.Logits(logits, **more)
        token, lp = torch.empty(n, dtype=torch.int32, device=dev), torch.empty(n, device=dev)
        draw = torch.empty(desc.scratch, device=dev)
        pg.pg_sample_tokens(desc, torch.full((n,), float(temperature), device=dev), seed, step, ids, token, lp, draw)
        undrawn |= (token < 0).any()
        drawn = token.clamp_min(0).long()
        logp[step, ids.long()] = lp
        score += (token_reward[drawn] - score) / (step + 1)
        history.scatter_(1, (n_prompt + step).long()[:, None], drawn.int()[:, None])
        if step in keep:                                 # checkpoint: the members whose rewards vary most go on
            k = keep[step]
            sel = torch.empty(P * k, dtype=torch.int32, device=dev)
            new_offsets = torch.empty(P + 1, dtype=torch.int32, device=dev)
            pg.pg_ovf_select(score, offsets, ints([k] * P), P, torch.empty(P, dtype=torch.int64, device=dev), sel, new_offsets, status,
                             torch.empty(pg.pg_ovf_scratch_ints(P), dtype=torch.int32, device=dev))
            table, lens = take(sel, table, lens)
            s = sel.long()
            ids, drawn, score, history, n_prompt, offsets = ids[s], drawn[s], score[s], history[s], n_prompt[s], new_offsets
        if step + 1 < steps:
            one = torch.ones_like(lens)
            pg.pg_cache_reserve(cache, table, lens, one, lens)
            logits = decoder.forward(drawn.int(), lens - 1, table, lens, lens)
    adv = torch.empty_like(score)
    pg.pg_group_advantages(score, offsets, P, adv_eps, adv)
    pg.pg_cache_check(cache)
    if undrawn:
        raise pg.PgError(pg.PG_EINVAL, "a member had no token to draw: a mask that allows none, or logits that are no numbers")
    if int(status[0]):
        raise pg.PgError(pg.PG_ENAN, "a non-finite proxy reward reached the selection")
    return dict(ids=ids, tokens=history, lens=n_prompt + steps, rewards=score, advantages=adv, logp=logp, offsets=offsets, penalties=penalties)


def _drawn(decoder, out):
    """Hidden states [survivors * steps, D] before every drawn token of sample_groups' survivors, and these tokens; clears the cache."""
    dev, cache, steps = out["tokens"].device, decoder.cache, out["logp"].shape[0]
    rows, sizes = out["tokens"].cpu().numpy(), out["lens"].cpu().numpy() - 1          # the last token is followed by none
    ints = lambda a: torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(dev)  # noqa: E731
    pg.pg_cache_clear(cache)
    table = torch.full((len(rows), decoder.width), -1, dtype=torch.int32, device=dev)
    lens = torch.zeros(len(rows), dtype=torch.int32, device=dev)
    pg.pg_cache_reserve(cache, table, lens, ints(sizes), lens)
    at = np.concatenate([np.arange(n) for n in sizes])
    hidden = decoder.hidden(ints(np.concatenate([r[:n] for r, n in zip(rows, sizes)])), ints(at), table, lens, ints(at + 1),
                            row_of=ints(np.repeat(np.arange(len(rows)), sizes)), cu=ints(np.cumsum([0] + sizes.tolist())))
    pg.pg_cache_check(cache)
    places = np.concatenate([end - steps + np.arange(steps) for end in np.cumsum(sizes)])
    drawn = np.concatenate([r[n + 1 - steps:n + 1] for r, n in zip(rows, sizes)])
    return hidden[torch.from_numpy(places).to(dev)].contiguous(), ints(drawn)


def _rows_of(logits, temperature, allow):
    """(logits with their mask, a temperature for each row)."""
    n, dev = logits.shape[0], logits.device
    more = {} if allow is None else dict(allow=allow, allow_row=torch.zeros(n, dtype=torch.int32, device=dev))
    return pg.Logits(logits, **more), torch.full((n,), float(temperature), device=dev)


def _without_penalties(out):
    """Raises ValueError for rollouts whose tokens were drawn from other logits than the decoder's."""
    if out.get("penalties") is not None and tuple(float(p) for p in out["penalties"]) != (1.0, 0.0, 0.0):
        raise ValueError(f"rollouts drawn with penalties {tuple(out['penalties'])}: their log-probs are not those of the decoder's own logits")


def token_logprobs(decoder, out, temperature=1.0, allow=None):
    """Log-probs of the drawn tokens of sample_groups' survivors under `decoder`'s weights, and entropies: [survivors, steps] each.  Clears the
    decoder's cache.  Temperature and mask as in sample_groups, which must not have had penalties (ValueError)."""
    _without_penalties(out)
    hidden, drawn = _drawn(decoder, out)
    desc, t = _rows_of(_linear(hidden, decoder.w["head"]), temperature, allow)
    logp, entropy = torch.empty(desc.rows, device=hidden.device), torch.empty(desc.rows, device=hidden.device)
    scratch = torch.empty(pg.pg_logprob_scratch_floats(desc.rows, desc.vocab), device=hidden.device)
    pg.pg_token_logprobs(desc, drawn, logp, scratch, temperature=t, entropy=entropy)
    return logp.view(out["ids"].shape[0], -1), entropy.view(out["ids"].shape[0], -1)


def policy_gradient(decoder, out, clip_low=0.2, clip_high=0.2, kl_coef=0.0, logp_ref=None, entropy_coef=0.0, temperature=1.0, allow=None):
    """The clipped objective of sample_groups' survivors under `decoder`'s weights, and its gradient, as far as the decoder's output matrix.

    Per sequence the mean over its drawn tokens, as pg_token_surrogate defines it, plus entropy_coef times the mean entropy; the gradient is that
    of the sequences' mean.  logp_ref: [survivors, steps] of a reference policy (token_logprobs).  Returns objective, kl, clipped [survivors],
    logp [survivors, steps], and with respect to what is maximised: d_logits [survivors * steps, vocab], hidden (what the logits were made of)
    and d_head = d_logits^T hidden.  Temperature and mask as in sample_groups, which must not have had penalties (ValueError)."""
    _without_penalties(out)
    hidden, drawn = _drawn(decoder, out)
    dev, n, steps = hidden.device, out["ids"].shape[0], out["logp"].shape[0]
    desc, t = _rows_of(_linear(hidden, decoder.w["head"]), temperature, allow)
    logits, empty = desc.keep[0], lambda *shape: torch.empty(*shape, device=dev)
    logp, stats, g = empty(n * steps), empty(n * steps, pg.PG_LOGPROB_STATS), empty(n * steps)
    pg.pg_token_logprobs(desc, drawn, logp, empty(pg.pg_logprob_scratch_floats(n * steps, desc.vocab)), temperature=t, stats=stats)
    old = out["logp"][:, out["ids"].long()].t().contiguous().view(-1)
    cu = torch.arange(0, n * steps + 1, steps, dtype=torch.int32, device=dev)
    objective, kl, clipped = empty(n), empty(n), torch.empty(n, dtype=torch.int32, device=dev)
    pg.pg_token_surrogate(logp, old, out["advantages"], cu, objective, g, clip_low, clip_high, steps, empty(pg.pg_surrogate_scratch_floats(n, steps)),
                          logp_ref=None if logp_ref is None else logp_ref.contiguous().view(-1), kl_coef=kl_coef, kl=kl, clipped=clipped)
    objective += entropy_coef * stats[:, 2].view(n, steps).mean(1)
    more = dict(g_entropy=torch.full_like(g, entropy_coef / (n * steps))) if entropy_coef else {}
    pg.pg_token_logprobs_backward(desc, drawn, stats, logits, g_logp=g / n, temperature=t, **more)           # in the logits' place
    return dict(objective=objective, kl=kl, clipped=clipped, logp=logp.view(n, steps), d_logits=logits, hidden=hidden, d_head=logits.t() @ hidden.float())


def distill_gradient(decoder, teacher, out, k=20, temperature=1.0, tail=True, allow=None):
    """The divergence of `decoder` from another decoder's k most likely tokens at every drawn token of sample_groups' survivors, and the gradient of
    its mean with respect to the decoder's output matrix, both from their own logits, whatever penalties the tokens were drawn with.  Returns loss [survivors, steps], d_logits, hidden and d_head."""
    hidden, drawn = _drawn(teacher, out)
    desc, t = _rows_of(_linear(hidden, teacher.w["head"]), temperature, allow)
    dev, n, vocab = hidden.device, desc.rows, desc.vocab
    ids, values = torch.empty(n, k, dtype=torch.int32, device=dev), torch.empty(n, k, device=dev)
    pg.pg_token_logprobs(desc, drawn, None, torch.empty(pg.pg_logprob_scratch_floats(n, vocab, k), device=dev), temperature=t, top_ids=ids, top_logp=values)
    hidden, _ = _drawn(decoder, out)
    desc, _ = _rows_of(_linear(hidden, decoder.w["head"]), temperature, allow)
    loss, stats, logits = torch.empty(n, device=dev), torch.empty(n, pg.PG_DISTILL_STATS, device=dev), desc.keep[0]
    pg.pg_distill_loss(desc, ids, values, loss, torch.empty(pg.pg_distill_scratch_floats(n, vocab), device=dev), tail=tail, temperature=t, stats=stats)
    pg.pg_distill_backward(desc, ids, values, stats, torch.full((n,), 1.0 / n, device=dev), logits, temperature=t)
    return dict(loss=loss.view(out["ids"].shape[0], -1), d_logits=logits, hidden=hidden, d_head=logits.t() @ hidden.float())


def main():
    cfg = SMALL
    rng = np.random.default_rng(MASTER_SEED)
    prompts = [rng.integers(0, cfg["vocab"], size=n).tolist() for n in (77, 26, 40)]
    reward = torch.from_numpy(rng.standard_normal(cfg["vocab"]).astype(np.float32)).to("cuda:0")
    decoder = Decoder(cfg, make_weights(cfg), rows=3 * 48)
    out = sample_groups(decoder, prompts, 48, 40, [(8, 32), (16, 16)], seed=1234, token_reward=reward, penalties=(1.1, 0.1, 0.0))
    for g in range(3):
        a, b = int(out["offsets"][g]), int(out["offsets"][g + 1])
        print(f"group {g}: {b - a} of 48 members, rewards' spread {float(out['rewards'][a:b].std(unbiased=False)):.3f}, "
              f"best member {int(out['ids'][a + int(out['advantages'][a:b].argmax())])} with advantage {float(out['advantages'][a:b].max()):.2f}")
    out = sample_groups(decoder, prompts, 48, 40, [(8, 32), (16, 16)], seed=1234, token_reward=reward)
    step = policy_gradient(decoder, out, entropy_coef=0.01)
    print(f"without penalties: objective {float(step['objective'].mean()):.4f}, {int(step['clipped'].sum())} of {step['logp'].numel()} tokens cut, "
          f"gradient of the output matrix {float(step['d_head'].norm()):.4f}")


if __name__ == "__main__":
    main()
