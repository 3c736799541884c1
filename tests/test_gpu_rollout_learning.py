"""What a token policy learns from its rollouts: draws, log-probs under the same and other weights, the objective and the distillation with their
gradients, through the library's calls together."""
import numpy as np
import pytest
import torch

from oracle import token_loss as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
CFG = dict(D=128, blocks=2, heads=4, kv_heads=2, vocab=508, page=16, max_len=128)
MEMBERS, STEPS, TEMPERATURE = 8, 12, 0.9


def f32(t):
    return t.detach().cpu().double().numpy()


@pytest.fixture(scope="module")
def rolled(lib):
    from paper_2512_15347_amd import rollout
    rng = np.random.default_rng(4)
    prompts = [rng.integers(0, CFG["vocab"], size=n).tolist() for n in (33, 1, 20)]
    reward = torch.from_numpy(rng.standard_normal(CFG["vocab"]).astype(np.float32)).to(DEV)
    words = -(-CFG["vocab"] // 32)
    allow = torch.full((1, words), -1, dtype=torch.int32, device=DEV)
    allow[0, 2:5] = 0x0F0F0F0F
    weights = rollout.make_weights(CFG, seed=9)
    decoder = rollout.Decoder(CFG, weights, rows=len(prompts) * MEMBERS)
    out = rollout.sample_groups(decoder, prompts, MEMBERS, STEPS, [(3, 5)], seed=77, token_reward=reward, temperature=TEMPERATURE, allow=allow)
    other = rollout.make_weights(CFG, seed=9)
    rs = torch.Generator().manual_seed(1)
    other["head"] = (other["head"].float().cpu() + 0.02 * torch.randn(other["head"].shape, generator=rs) * 4).to(torch.bfloat16).to(DEV)
    return rollout, decoder, rollout.Decoder(CFG, other, rows=len(prompts) * MEMBERS), out, allow


def open_tokens(allow):
    bits = np.unpackbits(allow.cpu().numpy().view(np.uint8), bitorder="little")[:CFG["vocab"]]
    return bits.astype(bool)


def test_the_rollouts_own_log_probs_come_out_again(rolled):
    rollout, decoder, _, out, allow = rolled
    logp, entropy = rollout.token_logprobs(decoder, out, temperature=TEMPERATURE, allow=allow)
    old = out["logp"][:, out["ids"].long()].t()
    assert logp.shape == (15, STEPS) and (entropy > 0).all()
    # the logits come from the same bf16 values, but sums of other lengths: a few roundings of values of about ten, some flipped bf16 roundings of
    # activations (2^-8 of one value of 128) in between
    assert float((logp - old).abs().max()) < 0.05
    step = rollout.policy_gradient(decoder, out, temperature=TEMPERATURE, allow=allow)
    want = torch.exp(logp - old).mul(out["advantages"][:, None]).mean(1)
    assert torch.equal(step["logp"], logp) and float((step["objective"] - want).abs().max()) < 1e-5 and int(step["clipped"].sum()) == 0


def objective(logits, out, logp_ref, allow, beta, entropy_coef):
    """Mean over the sequences in fp64, from logits [survivors * steps, vocab]."""
    n, total = out["ids"].shape[0], 0.0
    rows, lens, adv = out["tokens"].cpu().numpy(), out["lens"].cpu().numpy(), f32(out["advantages"])
    old = f32(out["logp"][:, out["ids"].long()].t())
    t = float(np.float32(TEMPERATURE))
    for r in range(n):
        drawn = rows[r, lens[r] - STEPS:lens[r]]
        each = [ref.token_logprobs(logits[r * STEPS + s], int(drawn[s]), t, allow) for s in range(STEPS)]
        logp = np.array([e["logp"] for e in each])
        total += ref.surrogate(logp, old[r], adv[r], 0.1, 0.15, None if logp_ref is None else logp_ref[r], beta)["objective"]
        total += entropy_coef * np.mean([e["entropy"] for e in each])
    return total / n


def test_the_gradient_of_the_output_matrix_against_differences(rolled):
    rollout, decoder, other, out, allow = rolled
    logp_ref, _ = rollout.token_logprobs(decoder, out, temperature=TEMPERATURE, allow=allow)
    beta, coef = 0.05, 0.01
    step = rollout.policy_gradient(other, out, 0.1, 0.15, beta, logp_ref, coef, TEMPERATURE, allow)
    assert int(step["clipped"].sum()) > 0 and (step["kl"] > 0).all()
    hidden, head, d_head = f32(step["hidden"]), f32(other.w["head"]), f32(step["d_head"])
    ref_logp, open_ = f32(logp_ref), open_tokens(allow)
    value = lambda w: objective(hidden @ w.T, out, ref_logp, open_, float(np.float32(beta)), coef)  # noqa: E731
    # fp32 logits of products of 128: 128 roundings of values of about ten
    assert abs(float(step["objective"].mean()) - value(head)) < 1e-3
    assert not d_head[~open_].any()
    rng = np.random.default_rng(2)
    for _ in range(3):
        way = rng.standard_normal(head.shape)
        h = 1e-6
        slope = (value(head + h * way) - value(head - h * way)) / (2 * h)
        assert abs(slope - np.sum(d_head * way)) < 2e-4 * np.sum(np.abs(d_head * way)) + 1e-8


def test_the_slope_along_the_gradient_is_its_squared_norm(rolled):
    rollout, decoder, _, out, allow = rolled
    step = rollout.policy_gradient(decoder, out, temperature=TEMPERATURE, allow=allow)
    hidden, head, d = f32(step["hidden"]), f32(decoder.w["head"]), f32(step["d_head"])
    args = out, None, open_tokens(allow), 0.0, 0.0
    at = lambda w: objective(hidden @ w.T, *args)  # noqa: E731
    size = 1e-3 / np.sum(d * d)
    gain = at(head + size * d) - at(head)
    assert abs(gain - 1e-3) < 2e-4                          # to first order the step times the squared norm


def test_distillation_of_a_decoder(rolled):
    rollout, decoder, other, out, allow = rolled
    same = rollout.distill_gradient(decoder, decoder, out, k=20, temperature=TEMPERATURE, allow=allow)
    assert float(same["loss"].abs().max()) < 1e-4 and float(same["d_logits"].abs().max()) < 1e-6
    step = rollout.distill_gradient(other, decoder, out, k=20, temperature=TEMPERATURE, allow=allow)
    assert (step["loss"] > 0).all()
    # against the definition, from the same hidden states
    t, open_ = float(np.float32(TEMPERATURE)), open_tokens(allow)
    hidden, head = f32(step["hidden"]), f32(other.w["head"])
    teacher = f32(same["hidden"]) @ f32(decoder.w["head"]).T
    loss, d = f32(step["loss"]).reshape(-1), f32(step["d_logits"])
    for r in (0, 50, 179):
        best = ref.token_logprobs(teacher[r], None, t, open_, 20)
        want, grad = ref.distill(hidden[r] @ head.T, best["top_ids"], best["top_logp"], True, t, open_)
        # logits of 128 products in fp32, twice
        assert abs(loss[r] - want) < 1e-4 * (1 + abs(want))
        assert np.max(np.abs(d[r] * 180 - grad)) < 1e-4


def test_what_does_not_fit_is_refused(rolled):
    rollout, decoder, other, out, allow = rolled
    with pytest.raises(AssertionError):
        rollout.policy_gradient(decoder, out, logp_ref=torch.zeros(15, STEPS + 1, device=DEV))
    from paper_2512_15347_amd import binding as pg
    with pytest.raises(pg.PgError):
        rollout.policy_gradient(decoder, out, clip_low=1.5)
    with pytest.raises(pg.PgError):
        rollout.distill_gradient(decoder, other, out, k=65)


def test_rollouts_say_what_penalties_they_were_drawn_with(rolled):
    rollout, decoder, _, out, _ = rolled
    assert out["penalties"] is None
    reward = torch.zeros(CFG["vocab"], device=DEV)
    drawn = [rollout.sample_groups(decoder, [[1, 2, 3]], 4, 3, [], seed=5, token_reward=reward, penalties=p) for p in ((1.3, 0.0, 0.2), (1.0, 0.0, 0.0), None)]
    for call in (rollout.token_logprobs, rollout.policy_gradient):
        with pytest.raises(ValueError):
            call(decoder, drawn[0])
    # penalties that change nothing: the draws and what is learnt from them are those without
    steps = [rollout.policy_gradient(decoder, o) for o in drawn[1:]]
    assert torch.equal(drawn[1]["tokens"], drawn[2]["tokens"]) and torch.equal(steps[0]["d_logits"], steps[1]["d_logits"])
    assert torch.isfinite(rollout.distill_gradient(decoder, decoder, drawn[0])["loss"]).all()
