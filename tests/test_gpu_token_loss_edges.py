"""What a token policy learns from, at the edges of what its calls allow: against the plain fp64 oracle, through the C ABI."""
import math

import numpy as np
import pytest
import torch

from oracle import token_loss as ref
from test_gpu_token_loss import DEV, TINY, U, Softmax, check_distill, check_logprobs, check_surrogate, dev, make_logits, mask_words, near, rounded, \
    run_distill, run_logprobs, run_surrogate, store_tol, teacher_lists

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n_top", [0, 5])
@pytest.mark.parametrize("rows,vocab", [(7, 3001), (7, 40001), (2500, 300)], ids=["one launch", "rows in pieces", "rows one after another"])
def test_rows_left_out_whose_temperature_is_none(lib, rows, vocab, n_top):
    """Padding: neither its logits nor its temperature reach an output."""
    rng = np.random.default_rng(rows + vocab)
    z = make_logits(rng, rows, vocab, False)
    target, t = rng.integers(0, vocab, size=rows), rng.uniform(0.6, 1.4, size=rows)
    t[:6] = [math.nan, -1.0, math.inf, math.nan, 1.0, -math.inf]
    target[[0, 1, 2, 4, 5]] = -1                           # of the rows without a temperature the fourth alone is not left out
    z[2] = math.nan
    g, ge = rng.standard_normal(rows), rng.standard_normal(rows)
    got = run_logprobs(lib, z, False, target, t, n_top=n_top, g=g, ge=ge)
    gone = target == -1
    assert not got["logp"][gone].any() and not got["entropy"][gone].any() and not got["d"][gone].any() and np.isnan(got["logp"][3])
    if n_top:
        assert (got["top_ids"][gone] == -1).all() and (got["top_logp"][gone] == -math.inf).all()
    check_logprobs(got, z, False, target, t, n_top=n_top, g=g, ge=ge)


@pytest.mark.parametrize("shift", [0.0, 1e3, -1e4, 1e5])
def test_a_shifted_list_has_the_same_gradient(lib, shift):
    """PG_DISTILL_TOP takes values up to a constant: rounded to fp32 they are the list, and nothing more is lost of them."""
    rng = np.random.default_rng(31)
    rows, vocab, k = 4, 3001, 64
    z = make_logits(rng, rows, vocab, False)
    ids, values = teacher_lists(rng, z, k)
    values = (values.astype(np.float64) + shift).astype(np.float32)
    g = np.ones(rows)
    got = run_distill(lib, z, False, ids, values, False, g)
    check_distill(got, z, False, ids, values, False, g)
    for r in range(rows):
        v = values[r].astype(np.float64)
        w = np.exp(v - v.max()) / np.exp(v - v.max()).sum()
        s = Softmax(z[r], 1.0, None)
        want = ref.distill(z[r], ids[r], v, False)[1][ids[r]]
        # q: differences to the largest and to the logarithm of the sum (at most ln k), rounded once each, and the exponential
        tol = s.p[ids[r]] * (s.p_rel[ids[r]] + 8 * U) + w * U * (2 * (v.max() - v) + 4 * math.log(k) + 8)
        near(got[1][r][ids[r]], want, tol + store_tol(want, False) + TINY, f"gradient of row {r}'s listed tokens")


def far_sequences(rng, lens, adv, distances):
    """Sequences near the old policy, some tokens of which are `distances` away from the old and from the reference policy."""
    seqs, refs = [], []
    for n, a in zip(lens, adv):
        logp = -np.abs(rng.standard_normal(n)) * 2
        old, x = logp + rng.standard_normal(n) * 0.1, logp + rng.standard_normal(n) * 0.2
        at = rng.integers(0, n, size=len(distances))
        x[at] = logp[at] + distances
        old[at[::2]] = logp[at[::2]] - np.asarray(distances)[::2]
        seqs.append((logp, old, a))
        refs.append(x)
    return seqs, refs


@pytest.mark.parametrize("lens", [[1, 5, 300], [5000, 70, 8192], [9000, 20000, 3]])
@pytest.mark.parametrize("kl_coef,adv,weight,distances", [
    (0.0, 0.7, None, [89.0, 120.0, 300.0]), (0.0, -1e-3, 2.0, [700.0, 1000.0, 41.0]), (1e-6, 1e-5, None, [89.0, 95.0, 60.0]),
    (1e-25, -1e-30, None, [130.0, 90.0, 89.0]), (0.05, -2.0, 1e-20, [100.0, 110.0, 95.0]), (0.1, 1e20, 1e-9, [39.0, 45.0, -60.0])])
def test_tokens_far_from_the_other_policies(lib, lens, kl_coef, adv, weight, distances):
    """Ratios and divergences that are no numbers of fp32 before they are scaled by what makes them some."""
    rng = np.random.default_rng(sum(lens))
    seqs, refs = far_sequences(rng, lens, [adv, -adv, adv], distances)
    w = None if weight is None else [weight] * 3
    for hi in (0.28, math.inf):
        got = run_surrogate(lib, seqs, 0.2, hi, refs=refs, kl_coef=kl_coef, weight=w)
        check_surrogate(got, seqs, 0.2, hi, refs, kl_coef, w)
        if kl_coef == 0.0 and adv > 0 and hi < 1:          # ratios above the bound are cut
            assert np.isfinite(got["objective"][[0, 2]]).all()


def test_the_divergence_can_be_watched_alone(lib):
    """kl_coef 0: a reference that is no number, or infinitely far away, reaches kl alone."""
    seqs = [([-1.0, -2.0], [-1.1, -2.0], 1.5), ([-1.0, -math.inf], [-1.0, -2.0], 1.0), ([-1.0], [-1.2], -1.0)]
    without = run_surrogate(lib, seqs, 0.2, 0.2)
    got = run_surrogate(lib, seqs, 0.2, 0.2, refs=[[-1.0, math.nan], [-1.0, -1.0], [-math.inf]], kl_coef=0.0)
    assert np.array_equal(got["clipped"], without["clipped"]) and np.isfinite(got["objective"]).all()
    for k in ("objective", "g_logp"):                      # a few roundings of one or two terms
        near(got[k], without[k], 16 * U * np.abs(without[k]), k)
    assert np.isnan(got["kl"][0]) and (got["kl"][1:] == math.inf).all()


def test_gradients_in_the_place_of_an_input(lib):
    """Of log-probs, old ones or the reference's: the same bits as apart, with gradients that would be far from anything if they were read as inputs."""
    rng = np.random.default_rng(8)
    lens = [800, 1, 1025, 300, 5000, 9000, 257] * 20
    cu = np.cumsum([0] + lens)
    n, seqs = int(cu[-1]), len(lens)
    logp = -np.abs(rng.standard_normal(n)) * 2
    old, x = logp + rng.standard_normal(n) * 0.2, logp + rng.standard_normal(n) * 0.3
    old[rng.integers(0, n, size=50)] -= 60.0               # and some that are far indeed
    adv, weight = dev(rng.standard_normal(seqs) * 1e5, np.float32), torch.ones(seqs, device=DEV)
    scratch = torch.empty(lib.pg_surrogate_scratch_floats(seqs, 9000), device=DEV)

    def run(place):
        t = dict(logp=dev(logp, np.float32), old=dev(old, np.float32), ref=dev(x, np.float32), apart=torch.empty(n, device=DEV))
        objective = torch.empty(seqs, device=DEV)
        lib.pg_token_surrogate(t["logp"], t["old"], adv, dev(cu, np.int32), objective, t[place], 0.2, math.inf, 9000, scratch, logp_ref=t["ref"], kl_coef=0.1,
                               weight=weight)
        return objective, t[place]

    want = run("apart")
    for place in ("logp", "old", "ref"):
        got = run(place)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]), place


def test_more_sequences_than_wide_workgroups_fit_a_grid(lib):
    """2^22 sequences, of which 1024 lanes each would be 2^32 in all: sequences of no tokens, of one and of many."""
    n = 1 << 22
    gen = torch.Generator(device=DEV).manual_seed(5)
    lens = (torch.rand(n, device=DEV, generator=gen) < 0.01).long()
    lens[0], lens[n // 2], lens[n - 1] = 2000, 300, 1500
    cu = torch.cat([torch.zeros(1, dtype=torch.long, device=DEV), lens.cumsum(0)])
    tokens = int(cu[-1])
    logp = -torch.rand(tokens, device=DEV, generator=gen)
    old, adv = logp + 0.1 * torch.randn(tokens, device=DEV, generator=gen), torch.randn(n, device=DEV, generator=gen)
    objective, g = torch.full((n,), 99.0, device=DEV), torch.full((tokens,), 99.0, device=DEV)
    assert lib.pg_surrogate_scratch_floats(n, 2000) == 0
    lib.pg_token_surrogate(logp, old, adv, cu.int(), objective, g, 1.0, math.inf, 2000)
    seq = torch.repeat_interleave(torch.arange(n, device=DEV), lens)
    ra = torch.exp(logp.double() - old.double()) * adv.double()[seq]
    want = torch.zeros(n, dtype=torch.float64, device=DEV).index_add_(0, seq, ra / lens[seq])
    # a lane adds at most 8 terms, 14 steps join the lanes, each term is off by some 12 roundings
    tol = torch.zeros(n, dtype=torch.float64, device=DEV).index_add_(0, seq, ra.abs() / lens[seq]) * 40 * U
    assert ((objective.double() - want).abs() <= tol).all()
    assert ((g.double() - ra / lens[seq]).abs() <= 16 * U * (ra / lens[seq]).abs()).all()


TEMPERATURES = [1e-3, 1e-12, 1e-20, 3e-25, 1e-30, 2e-38, 1e-39, 1e-44, 1e6, 1e12, 1e20, 1e30, 1e36, 1e37, 3e38]


def logits_for(rng, t, vocab, bf):
    """Of a few temperatures, above 1; or ordinary ones, of which one or few equal ones remain."""
    if t > 1:
        return np.clip(rng.standard_normal(vocab) * 2.0 * t, -3.3e38, 3.3e38)
    z = rng.standard_normal(vocab) * 3
    z[rng.integers(0, vocab, size=3)] = z.max()
    return z


def extreme_rows(rng, bf, vocab):
    t = np.array(TEMPERATURES, dtype=np.float32)
    z = rounded(np.stack([logits_for(rng, float(v), vocab, bf) for v in t]), bf)
    return t, z


def with_holes(rng, z, target):
    """Masks that leave the targets, and logits of -inf."""
    open_ = rng.random(z.shape) < 0.8
    open_[np.arange(len(z)), target] = True
    z[:, 3::7] = -math.inf
    return open_


def targets(rng, z):
    target = rng.integers(0, z.shape[1], size=len(z))
    target[::2] = z[::2].argmax(1)
    return target


@pytest.mark.parametrize("holes", [False, True], ids=["whole", "holes"])
@pytest.mark.parametrize("bf", [False, True], ids=["f32", "bf16"])
@pytest.mark.parametrize("vocab", [70, 3001, 33000])
def test_every_temperature_gives_numbers(lib, vocab, bf, holes):
    """From the smallest number to nearly the largest, with logits of -inf and masks or without."""
    rng = np.random.default_rng(vocab)
    t, z = extreme_rows(rng, bf, vocab)
    target = targets(rng, z)
    open_ = with_holes(rng, z, target) if holes else None
    for n_top in (0, 5):
        got = run_logprobs(lib, z, bf, target, t, open_, None, n_top)
        check_logprobs(got, z, bf, target, t, open_, None, n_top)
        assert not np.isnan(got["logp"]).any() and not np.isnan(got["entropy"]).any()


@pytest.mark.parametrize("holes", [False, True], ids=["whole", "holes"])
@pytest.mark.parametrize("bf", [False, True], ids=["f32", "bf16"])
@pytest.mark.parametrize("vocab", [70, 3001, 33000])
def test_every_temperature_has_gradients(lib, vocab, bf, holes):
    """Of log-probs and entropies together, and of each alone."""
    rng = np.random.default_rng(vocab)
    t, z = extreme_rows(rng, bf, vocab)
    rows, target = len(t), targets(rng, z)
    open_ = with_holes(rng, z, target) if holes else None
    g, ge = rng.standard_normal(rows), rng.standard_normal(rows) * 0.3
    for a, b in ((g, ge), (g, None), (np.zeros(rows), ge)):
        got = run_logprobs(lib, z, bf, target, t, open_, None, 0, a, b)
        check_logprobs(got, z, bf, target, t, open_, None, 0, a, b)
        assert not np.isnan(got["d"]).any()


@pytest.mark.parametrize("holes", [False, True], ids=["whole", "holes"])
@pytest.mark.parametrize("bf", [False, True], ids=["f32", "bf16"])
@pytest.mark.parametrize("vocab", [70, 3001, 33000])
def test_distillation_at_every_temperature(lib, vocab, bf, holes):
    rng = np.random.default_rng(vocab + 1)
    t, z = extreme_rows(rng, bf, vocab)
    rows, k = len(t), 20
    if holes:
        z[:, 3::7] = -math.inf
    ids = np.stack([rng.permutation(np.flatnonzero(row > -math.inf))[:k] for row in z]).astype(np.int32)
    ids[::2, 0] = z[::2].argmax(1)
    ids[::2, 1:] = np.where(ids[::2, 1:] == ids[::2, :1], -1, ids[::2, 1:])
    values = np.log(rng.dirichlet(np.ones(k + 1), size=rows)[:, :k])
    g = rng.standard_normal(rows) * 100
    check_distill(run_distill(lib, z, bf, ids, values, False, g, t), z, bf, ids, values, False, g, t)
    # what is not listed has some of the mass above 1, where the logits are of that size
    warm = t > 1
    args = z[warm], bf, ids[warm], values[warm], True, g[warm], t[warm]
    check_distill(run_distill(lib, *args), *args)


@pytest.mark.parametrize("bf", [False, True], ids=["f32", "bf16"])
@pytest.mark.parametrize("vocab", [300, 9001, 40001])
def test_no_log_prob_is_above_0_and_no_entropy_below(lib, vocab, bf):
    """Rows of which one token has all of the mass, at any logit and temperature."""
    rng = np.random.default_rng(vocab)
    rows = 200
    z = np.full((rows, vocab), -1e4)
    target = rng.integers(0, vocab, size=rows)
    z[np.arange(rows), target] = rng.uniform(-30, 30, size=rows)
    z, t = rounded(z, bf), rng.uniform(0.3, 3.0, size=rows)
    got = run_logprobs(lib, z, bf, target, t, n_top=2)
    assert (got["logp"] <= 0).all() and (got["entropy"] >= 0).all() and (got["top_logp"] <= 0).all()
    check_logprobs(got, z, bf, target, t, n_top=2)


@pytest.mark.parametrize("value", [math.nan, math.inf])
@pytest.mark.parametrize("vocab", [20, 3000, 20000])
def test_a_bad_row_is_loud_whatever_its_list_says(lib, vocab, value):
    """The list has every token that is allowed, and gives none of them any weight."""
    rng = np.random.default_rng(vocab)
    z = make_logits(rng, 3, vocab, False)
    k = 20
    ids = np.stack([rng.permutation(vocab)[:k] for _ in range(3)]).astype(np.int32)
    open_ = np.zeros((3, vocab), dtype=bool)
    open_[np.arange(3)[:, None], ids] = True
    z[1, ids[1, 7]] = value
    values, g = np.full((3, k), -math.inf), np.ones(3)
    got = run_distill(lib, z, False, ids, values, True, g, None, open_, np.arange(3))
    assert np.isnan(got[0][1]) and got[0][[0, 2]].tolist() == [0, 0]
    check_distill(got, z, False, ids, values, True, g, None, open_, np.arange(3))


@pytest.mark.parametrize("bf", [False, True], ids=["f32", "bf16"])
@pytest.mark.parametrize("rows,vocab", [(3, 1000), (48, 16384), (5, 70001)])
def test_a_drawn_tokens_log_prob_is_the_draws(lib, rows, vocab, bf):
    """pg_token_logprobs of what pg_sample_tokens drew, from the same logits, temperatures and masks."""
    rng = np.random.default_rng(rows)
    z = make_logits(rng, rows, vocab, bf)
    t = rng.uniform(0.5, 1.5, size=rows)
    t[0] = 0.0
    open_ = rng.random((rows, vocab)) < 0.7
    logits = dev(z, np.float32).to(torch.bfloat16 if bf else torch.float32)
    desc, temperature = lib.Logits(logits, allow=dev(mask_words(open_), np.int32)), dev(t, np.float32)
    token, drawn, logp = torch.empty(rows, dtype=torch.int32, device=DEV), torch.empty(rows, device=DEV), torch.empty(rows, device=DEV)
    lib.pg_sample_tokens(desc, temperature, 5, 0, None, token, drawn, torch.empty(desc.scratch, device=DEV))
    lib.pg_token_logprobs(desc, token, logp, torch.empty(lib.pg_logprob_scratch_floats(rows, vocab), device=DEV), temperature=temperature)
    for r in range(rows):
        s = Softmax(z[r], float(np.float32(t[r])), open_[r])
        v = int(token[r])
        # each of the two is off by what the sums' and the logit's roundings allow
        assert open_[r, v] and abs(float(drawn[r]) - float(logp[r])) <= 2 * s.logp_tol(v) + 8 * U * abs(s.y.max())
