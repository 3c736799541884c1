"""The token policy's funnel as a whole: prompts, expansion, draws, prunes, advantages through the library's calls together."""
import math

import numpy as np
import pytest
import torch

from oracle import ovf

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
CFG = dict(D=128, blocks=2, heads=4, kv_heads=2, vocab=500, page=16, max_len=128)
MEMBERS, STEPS, SCHEDULE = 12, 24, [(3, 8), (15, 5)]


@pytest.fixture(scope="module")
def runs(lib):
    from paper_2512_15347_amd import rollout
    rng = np.random.default_rng(4)
    prompts = [rng.integers(0, CFG["vocab"], size=n).tolist() for n in (33, 1, 48, 70)]
    reward = torch.from_numpy(rng.standard_normal(CFG["vocab"]).astype(np.float32)).to(DEV)
    weights = rollout.make_weights(CFG, seed=9)
    print("token policy: pruned and unpruned runs", flush=True)
    out = []
    for schedule in (SCHEDULE, []):
        decoder = rollout.Decoder(CFG, weights, rows=len(prompts) * MEMBERS)
        r = rollout.sample_groups(decoder, prompts, MEMBERS, STEPS, schedule, seed=77, token_reward=reward, temperature=0.9,
                                  penalties=(1.2, 0.1, 0.2))
        torch.cuda.synchronize()
        held = int(decoder.cache.refs.sum())
        out.append((r, held))
    return prompts, reward.cpu().numpy(), weights, out


def test_survivors_do_not_depend_on_what_was_pruned(runs):
    prompts, reward, _, ((pruned, _), (full, _)) = runs
    ids = pruned["ids"].long()
    assert pruned["offsets"].tolist() == [0, 5, 10, 15, 20] and [int(i) // MEMBERS for i in ids] == sum([[g] * 5 for g in range(4)], [])
    assert torch.equal(pruned["tokens"], full["tokens"][ids])
    # the log-probs' sums are cut by the number of rows: some roundings of values of about 10
    assert float((pruned["logp"][:, ids] - full["logp"][:, ids]).abs().max()) < 1e-5
    gone = torch.isnan(pruned["logp"]).cpu().numpy()
    assert not gone[:4].any() and (gone[4:16].sum(1) == 4 * 4).all() and (gone[16:].sum(1) == 4 * 7).all()
    for r in range(20):
        g, n = int(ids[r]) // MEMBERS, int(pruned["lens"][r])
        row = pruned["tokens"][r, :n].cpu().numpy()
        assert row[:len(prompts[g])].tolist() == prompts[g]
        want = reward[row[len(prompts[g]):]].astype(np.float64).mean()
        assert abs(float(pruned["rewards"][r]) - want) < 1e-5


def test_the_survivors_of_the_first_checkpoint_are_the_filters(runs):
    """The unpruned run's drawn tokens give the rewards that the pruned one saw at its first checkpoint."""
    prompts, reward, _, ((pruned, _), (full, _)) = runs
    tokens = full["tokens"].cpu().numpy()
    score = np.zeros(len(tokens), dtype=np.float32)
    for r, row in enumerate(tokens):
        p = len(prompts[r // MEMBERS])
        for s in range(4):
            score[r] += (reward[row[p + s]] - score[r]) / np.float32(s + 1)
    offsets = np.arange(5) * MEMBERS
    _, sel, _ = ovf.ovf_groups(score, offsets, np.full(4, 8))
    alive = np.flatnonzero(~torch.isnan(pruned["logp"][4]).cpu().numpy())
    assert alive.tolist() == sel.tolist()


def test_pages_are_held_by_survivors_alone(runs):
    prompts, _, _, ((pruned, held), (full, held_full)) = runs
    # a row holds the pages of its prompt and of all drawn tokens but the last
    pages = lambda n: -(-n // CFG["page"])  # noqa: E731
    want = lambda k: sum(k * pages(len(p) + STEPS - 1) for p in prompts)  # noqa: E731
    assert held == want(5) and held_full == want(MEMBERS)


def test_log_probs_against_the_whole_sequence_in_64_bits(runs):
    prompts, _, weights, ((pruned, _), _) = runs
    bf = lambda x: x.float().to(torch.bfloat16).double()  # noqa: E731
    hd, group = CFG["D"] // CFG["heads"], CFG["heads"] // CFG["kv_heads"]
    w = {k: v.cpu().double() for k, v in weights.items() if k != "blocks"}
    blocks = [{k: v.cpu().double() for k, v in b.items()} for b in weights["blocks"]]
    norm = lambda x: bf(x / torch.sqrt(x.square().mean(1, keepdim=True) + 1e-6))  # noqa: E731
    for r in (0, 6, 11, 19):
        i, n = int(pruned["ids"][r]), int(pruned["lens"][r])
        row, p = pruned["tokens"][r, :n].cpu().long(), len(prompts[int(pruned["ids"][r]) // MEMBERS])
        x = w["embed"][row] + w["position"][:n]
        causal = torch.full((n, n), -math.inf, dtype=torch.float64).triu(1)
        for b in blocks:
            qkv = bf(norm(x) @ b["qkv"].T).view(n, -1, hd)
            heads = []
            for h in range(CFG["heads"]):
                q, k, v = qkv[:, h], qkv[:, CFG["heads"] + h // group], qkv[:, CFG["heads"] + CFG["kv_heads"] + h // group]
                heads.append(torch.softmax(q @ k.T / math.sqrt(hd) + causal, 1) @ v)
            x = x + bf(torch.cat(heads, 1)) @ b["o"].T
            x = x + bf(torch.nn.functional.gelu(norm(x) @ b["fc1"].T, approximate="tanh")) @ b["fc2"].T
        logits = norm(x) @ w["head"].T
        for s in range(STEPS):
            z = logits[p + s - 1].clone()
            seen, made = row[:p + s], row[p:p + s]
            z[seen] = torch.where(z[seen] > 0, z[seen] / 1.2, z[seen] * 1.2)
            count = torch.bincount(made, minlength=CFG["vocab"])
            z = (z - 0.1 * count - 0.2 * (count > 0)) / 0.9
            want = float(torch.log_softmax(z, 0)[row[p + s]])
            # logits from bf16 activations: 2e-2 of the largest, the network's own bound; they enter twice (the token's and the sum's)
            assert abs(float(pruned["logp"][s, i]) - want) <= 2 * 2e-2 * float(logits[p + s - 1].abs().max()) * 1.2 / 0.9, (r, s)


def test_a_grammar_mask_and_refusals(lib):
    from paper_2512_15347_amd import rollout
    weights = rollout.make_weights(CFG, seed=9)
    reward = torch.ones(CFG["vocab"], device=DEV)
    words = -(-CFG["vocab"] // 32)
    allow = torch.zeros(1, words, dtype=torch.int32, device=DEV)
    allow[0, 3] = 0b1011                                  # tokens 96, 97 and 99
    decoder = rollout.Decoder(CFG, weights, rows=4)
    out = rollout.sample_groups(decoder, [[5, 6]], 4, 6, [], 1, reward, allow=allow)
    assert set(out["tokens"][:, 2:].flatten().tolist()) <= {96, 97, 99}
    assert torch.isfinite(out["logp"]).all() and (out["logp"] <= 1e-6).all()
    with pytest.raises(ValueError):
        rollout.sample_groups(decoder, [[]], 4, 6, [], 1, reward)
    with pytest.raises(ValueError):
        rollout.sample_groups(decoder, [[1]], 4, 6, [(1, 5)], 1, reward)
    with pytest.raises(ValueError):
        rollout.sample_groups(decoder, [[1] * 100], 4, 60, [], 1, reward)
