"""GPU parity of what a token policy learns from against the plain fp64 oracle, through the C ABI.

Tolerances.  u = 2^-24.  1 / T, the product with z - m and the exponential round y - top at most four times, so a weight of the softmax is
off by u (4 |y - top| + 4) of itself; a lane adds at most vocab / 256 terms one after another and some 64 steps join the lanes and pieces, so a sum
of positive terms is off by (vocab / 256 + 64) u of itself.  The rest is what these two make of the formulas."""
import math

import numpy as np
import pytest
import torch

from oracle import token_loss as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
TINY = 2.0 ** -120                                       # below it results may be 0


def say(msg):
    print(msg, flush=True)


def dev(a, dtype):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=dtype)).to(DEV)


def rounded(x, bf):
    """What lies there, in fp64."""
    t = torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32))
    return (t.to(torch.bfloat16) if bf else t).double().numpy()


def place(z, bf, stride=None, offset=0, fill=7.0):
    """z in device rows `stride` apart, the first `offset` elements into its buffer; (rows, whole buffer)."""
    rows, vocab = z.shape
    stride = stride or vocab
    whole = torch.full((offset + rows * stride + 5,), fill, dtype=torch.bfloat16 if bf else torch.float32, device=DEV)
    view = whole[offset:offset + rows * stride].view(rows, stride)[:, :vocab]
    view.copy_(torch.from_numpy(np.ascontiguousarray(z, dtype=np.float32)).to(DEV))
    return view, whole


def mask_words(open_):
    m, vocab = open_.shape
    bits = np.zeros((m, -(-vocab // 32) * 32), dtype=np.uint8)
    bits[:, :vocab] = open_
    return np.packbits(bits, axis=1, bitorder="little").view(np.uint32).view(np.int32)


class Softmax:
    """What the tolerances of a row need."""

    def __init__(self, z, t, allow):
        self.y, self.ln, self.lse, self.bad = ref.softmax(z, t, allow)
        self.ok = not self.bad and self.lse > -np.inf
        if self.ok:
            self.p = np.exp(self.ln)
            self.far = np.where(self.p > 0, self.y.max() - self.y, 0.0)          # |y - top|
            mean, square = np.sum(self.p * self.far), np.sum(self.p * self.far ** 2)
            self.ln_s = -self.ln[np.argmax(self.y)]
            self.sum_tol = (len(z) / 256 + 64) * U
            self.lse_tol = self.sum_tol + U * (4 * mean + 4 + 2 * abs(self.ln_s))
            self.h = self.ln_s + mean
            self.h_tol = self.lse_tol + mean * (2 * self.sum_tol + 8 * U) + 4 * U * square + 2 * U * abs(self.h)
            self.p_rel = U * (4 * self.far + 8) + self.lse_tol

    def logp_tol(self, v):
        return self.lse_tol + 4 * U * self.far[v] + 2 * U * abs(self.ln[v])


def near(got, want, tol, what):
    got, want = np.asarray(got, dtype=np.float64), np.asarray(want, dtype=np.float64)
    want = np.where(np.abs(want) >= 2.0 ** 128, np.copysign(np.inf, want), want)        # no number of fp32
    same = (got == want) | (np.isnan(got) & np.isnan(want))
    fine = np.isfinite(got) & np.isfinite(want)
    off = np.zeros(got.shape)
    off[fine] = np.abs(got[fine] - want[fine]) - np.broadcast_to(tol, got.shape)[fine]
    wrong = ~same & (~fine | (off > 0))
    assert not wrong.any(), f"{what}: {int(wrong.sum())} wrong, first at {np.argwhere(wrong)[0].tolist()}: {got[wrong][0]!r}, wanted {want[wrong][0]!r}, " \
                            f"tolerance {np.broadcast_to(tol, got.shape)[wrong][0]!r}"


def store_tol(want, bf):
    return np.abs(want) * (2.0 ** -8 if bf else U) + (2.0 ** -133 if bf else 2.0 ** -149)


def make_logits(rng, rows, vocab, bf, scale=3.0):
    z = rng.standard_normal((rows, vocab)) * scale
    return rounded(z, bf)


def run_logprobs(lib, z, bf, target, temperature=None, open_=None, allow_row=None, n_top=0, g=None, ge=None, stride=None, offset=0, in_place=False):
    rows, vocab = z.shape
    logits, whole = place(z, bf, stride, offset)
    more = {}
    if open_ is not None:
        more = dict(allow=dev(mask_words(open_), np.int32), allow_row=None if allow_row is None else dev(allow_row, np.int32))
    desc = lib.Logits(logits, **more)
    f = lambda *s: torch.full(s, 99.0, device=DEV)  # noqa: E731
    out = dict(logp=f(rows), entropy=f(rows), stats=f(rows, lib.PG_LOGPROB_STATS))
    if n_top:
        out.update(top_ids=torch.full((rows, n_top), 99, dtype=torch.int32, device=DEV), top_logp=f(rows, n_top))
    scratch = torch.full((max(1, lib.pg_logprob_scratch_floats(rows, vocab, n_top)),), math.nan, device=DEV)
    t = None if temperature is None else dev(temperature, np.float32)
    tg = dev(target, np.int32)
    lib.pg_token_logprobs(desc, tg, out["logp"], scratch, temperature=t, **{k: v for k, v in out.items() if k != "logp"})
    if g is not None:
        if in_place:
            d, d_whole = logits, whole
        else:
            d, d_whole = place(np.full(z.shape, 5.0), bf, stride, (offset + 3) % 8 if offset else 0)
        lib.pg_token_logprobs_backward(desc, tg, out["stats"], d, g_logp=None if g is None else dev(g, np.float32),
                                       g_entropy=None if ge is None else dev(ge, np.float32), temperature=t)
        out["d"] = d.double()
        gaps = torch.ones(d_whole.shape, dtype=torch.bool, device=DEV)
        first = (d.data_ptr() - d_whole.data_ptr()) // d_whole.element_size()
        gaps.as_strided(d.shape, d.stride(), first).fill_(False)
        assert (d_whole[gaps] == 7.0).all(), "something beside the rows was written"
    torch.cuda.synchronize()
    return {k: v.cpu().numpy() for k, v in out.items()}


def check_logprobs(got, z, bf, target, temperature=None, open_=None, allow_row=None, n_top=0, g=None, ge=None):
    rows, vocab = z.shape
    for r in range(rows):
        t = 1.0 if temperature is None else float(np.float32(temperature[r]))
        allow = None
        if open_ is not None:
            m = r if allow_row is None else allow_row[r]
            allow = None if m == -1 else open_[m] if 0 <= m < len(open_) else np.zeros(vocab, dtype=bool)
        want = ref.token_logprobs(z[r], int(target[r]), t, allow, n_top)
        s = Softmax(z[r], t, allow)
        here = s.ok and target[r] != -1
        tol = s.logp_tol(target[r]) if here and 0 <= target[r] < vocab and want["logp"] > -np.inf else 0.0
        near(got["logp"][r], want["logp"], tol, f"logp of row {r}")
        near(got["entropy"][r], want["entropy"], s.h_tol if here else 0.0, f"entropy of row {r}")
        if target[r] != -1:
            lse = float(got["stats"][r, 0]) + float(got["stats"][r, 1])
            near(lse, want["lse"], s.lse_tol + 2 * U * abs(s.y.max()) if here else 0.0, f"denominator of row {r}")
        if n_top:
            assert got["top_ids"][r].tolist() == want["top_ids"].tolist(), f"alternatives of row {r}"
            ids = want["top_ids"]
            tol = np.array([s.logp_tol(i) if here and i >= 0 else 0.0 for i in ids])
            near(got["top_logp"][r], want["top_logp"], tol, f"log-probs of alternatives of row {r}")
        if g is not None:
            a, b = float(np.float32(g[r])), 0.0 if ge is None else float(np.float32(ge[r]))
            d = ref.token_logprobs_gradient(z[r], int(target[r]), a, b, t, allow)
            tol = 0.0
            if here:
                inv = 1.0 if t == 0 else 1 / t
                coef = abs(a) + abs(b) * (abs(s.h - s.ln_s) + s.far)
                tol = s.p * inv * (coef * (s.p_rel + 8 * U) + abs(b) * (s.h_tol + s.lse_tol)) + TINY * inv * (coef + 1)
                if 0 <= target[r] < vocab:
                    tol[target[r]] += 4 * U * abs(a) * inv
                tol = tol * (1 + 2.0 ** -7) + store_tol(d, bf)
            near(got["d"][r], d, tol, f"gradient of row {r}")


SIZES = [(1, 1), (3, 2), (2, 7), (5, 8), (4, 9), (3, 63), (2, 64), (3, 65), (2, 257), (2, 2047), (2, 2048), (3, 2049), (2, 8191), (1, 8193),
         (5, 16384), (2, 24001), (1, 65537), (2, 131073)]


@pytest.mark.parametrize("bf", [False, True], ids=["f32", "bf16"])
@pytest.mark.parametrize("rows,vocab", SIZES)
def test_logprobs_and_gradient(lib, rows, vocab, bf):
    rng = np.random.default_rng(rows * 1000 + vocab)
    z = make_logits(rng, rows, vocab, bf)
    target = rng.integers(0, vocab, size=rows)
    temperature = rng.uniform(0.5, 1.7, size=rows)
    temperature[rows // 2] = 0.0                           # taken at temperature 1, as the drawn token's log-prob is
    g, ge = rng.standard_normal(rows), rng.standard_normal(rows) * 0.3
    for n_top, place_as in ((0, {}), (1, dict(stride=vocab + 5, offset=1)), (20, dict(in_place=True)), (64, dict(offset=3))):
        got = run_logprobs(lib, z, bf, target, temperature, n_top=n_top, g=g, ge=ge, **place_as)
        check_logprobs(got, z, bf, target, temperature, n_top=n_top, g=g, ge=ge)


@pytest.mark.parametrize("bf", [False, True], ids=["f32", "bf16"])
@pytest.mark.parametrize("vocab", [5, 64, 1000, 2049, 16385, 40001])
def test_masks_and_rows_left_out(lib, vocab, bf):
    rng = np.random.default_rng(vocab)
    rows = 14
    z = make_logits(rng, rows, vocab, bf)
    open_ = rng.random((4, vocab)) < np.array([0.5, 0.05, 0.97, 0.0])[:, None]
    open_[1, :] = False
    open_[1, vocab // 2] = True                            # one token
    if vocab > 4000:
        open_[0, 1000:3500] = False                        # a long run
    allow_row = np.array([0, 1, 2, 3, -1, 0, 2, 7, -5, 0, 1, -1, 2, 0])
    target = rng.integers(0, vocab, size=rows)
    for r in range(rows):
        m = allow_row[r]
        if 0 <= m < 4 and open_[m].any() and r != 12:
            target[r] = np.flatnonzero(open_[m])[r % open_[m].sum()]
    if not open_[2].all():
        target[12] = np.flatnonzero(~open_[2])[0]          # a token that is not allowed: -inf
    target[5], target[6], target[11] = -1, vocab, -2       # left out, and two that no token has
    g, ge = rng.standard_normal(rows), rng.standard_normal(rows)
    g[9] = ge[9] = 0.0
    for n_top in (0, 64):
        got = run_logprobs(lib, z, bf, target, None, open_, allow_row, n_top, g, ge)
        check_logprobs(got, z, bf, target, None, open_, allow_row, n_top, g, ge)
    # a mask for every row
    some = rng.random((rows, vocab)) < 0.6
    got = run_logprobs(lib, z, bf, target, None, some, None, 5, g, None, stride=vocab + 1)
    check_logprobs(got, z, bf, target, None, some, None, 5, g, None)


@pytest.mark.parametrize("bf", [False, True], ids=["f32", "bf16"])
@pytest.mark.parametrize("vocab", [3, 70, 4097, 33000])
def test_infinities_nan_and_lowest_values(lib, vocab, bf):
    rng = np.random.default_rng(vocab + 1)
    lowest = float(torch.finfo(torch.bfloat16 if bf else torch.float32).min)
    z = make_logits(rng, 14, vocab, bf)
    at = vocab // 2
    z[0] = -np.inf                                         # nothing left
    z[1, at:] = -np.inf
    z[2] = lowest                                          # all equally likely
    z[3, 1:] = lowest
    z[4, at] = np.nan
    z[5, at] = np.inf
    z[6] = -np.inf
    z[6, at] = -3.0                                        # one token
    z[7, at] = -lowest                                     # the largest number
    z[7, 0] = lowest
    z[8] = 0.0
    z[9] = rounded(z[9] + 30000.0, bf)                     # shifted far
    z[10] = rounded(z[10] * 1e30, bf)
    z[11] = np.inf
    z[12], z[13] = np.nan, rounded(z[13] * 1e-30, bf)
    target = np.full(14, at)
    target[1] = vocab - 1                                  # a token of -inf
    g, ge = rng.standard_normal(14), rng.standard_normal(14)
    for n_top in (0, 20):
        got = run_logprobs(lib, z, bf, target, None, n_top=n_top, g=g, ge=ge)
        check_logprobs(got, z, bf, target, None, n_top=n_top, g=g, ge=ge)


@pytest.mark.parametrize("bf", [False, True], ids=["f32", "bf16"])
@pytest.mark.parametrize("value", ["lowest", "-inf"])
def test_long_runs_that_an_added_mask_has_left(lib, value, bf):
    """Whole passes, waves and pieces of the type's lowest value, or of -inf, before, between and behind the other logits."""
    rng = np.random.default_rng(21)
    vocab, low = 40003, float(torch.finfo(torch.bfloat16 if bf else torch.float32).min) if value == "lowest" else -np.inf
    z = make_logits(rng, 6, vocab, bf)
    z[0, :20000] = low
    z[1, 300:] = low
    z[2, :39000] = z[2, 39900:] = low
    z[3, 2000:30000] = low
    z[4, ::3] = low
    z[5, np.arange(vocab) // 8 % 64 < 40] = low            # some lanes of every wave
    target = np.array([30000, 5, 39500, 1, 7, 40 * 8])
    g, ge = rng.standard_normal(6), rng.standard_normal(6)
    check_logprobs(run_logprobs(lib, z, bf, target, None, n_top=64, g=g, ge=ge), z, bf, target, None, n_top=64, g=g, ge=ge)
    # and of rows that are a workgroup's each, several of them one after another
    rows = np.tile(z[:, :9000], (500, 1))
    got = run_logprobs(lib, rows, bf, np.tile(target % 9000, 500), None, n_top=3, g=np.tile(g, 500), ge=np.tile(ge, 500))
    for k in ("logp", "entropy", "top_ids", "d"):          # a row's parts depend on its place: some roundings
        a, b = np.where(np.isfinite(got[k]), got[k], -1e4).astype(np.float64), got[k].reshape((500, 6) + got[k].shape[1:])
        first = np.tile(a[:6], (500,) + (1,) * (a.ndim - 1))
        assert np.allclose(a, first, rtol=2 ** -6 if k == "d" else 1e-5, atol=1e-6 if k != "d" else 1e-7), k
    check_logprobs({k: v[-6:] for k, v in got.items()}, rows[-6:], bf, (target % 9000), None, n_top=3, g=g, ge=ge)
    ids, values = teacher_lists(rng, np.where(z == low, -30.0, z), 30)
    t = np.array([1.0, 0.7, 1.3, 1.0, 1.0, 1.0])
    check_distill(run_distill(lib, z, bf, ids, values, True, g, t), z, bf, ids, values, True, g, t)


@pytest.mark.parametrize("bf", [False, True], ids=["f32", "bf16"])
def test_rows_that_are_left_out_are_not_read(lib, bf):
    z = np.full((4, 5001), np.nan)
    z[2] = rounded(np.random.default_rng(1).standard_normal(5001), bf)
    target = np.array([-1, 3, 4, -1])
    got = run_logprobs(lib, z, bf, target, None, n_top=2, g=np.array([1.0, 0.0, 1.0, 2.0]), ge=np.array([1.0, 0.0, 0.0, 1.0]))
    assert not got["d"][[0, 1, 3]].any() and np.isfinite(got["d"][2]).all() and got["logp"][[0, 3]].tolist() == [0, 0] and np.isnan(got["logp"][1])
    assert got["entropy"][[0, 3]].tolist() == [0, 0] and (got["top_ids"][[0, 1, 3]] == -1).all() and np.isnan(got["top_logp"][1]).all()
    ids, values = np.full((4, 3), -1), np.zeros((4, 3))
    ids[1:3], values[1:3] = [1, 2, 3], -2.0
    loss, d = run_distill(lib, z, bf, ids, values, True, np.array([1.0, 0.0, 1.0, 1.0]))
    assert not d[[0, 1, 3]].any() and loss[[0, 3]].tolist() == [0, 0] and np.isnan(loss[1]) and np.isfinite(loss[2])


def test_temperatures_that_are_none(lib):
    rng = np.random.default_rng(8)
    z = make_logits(rng, 6, 3001, False)
    target = np.arange(6)
    t = np.array([-1.0, np.inf, np.nan, -0.0, 1e-3, 50.0])
    g = np.ones(6)
    got = run_logprobs(lib, z, False, target, t, n_top=3, g=g)
    check_logprobs(got, z, False, target, t, n_top=3, g=g)


@pytest.mark.parametrize("bf", [False, True], ids=["f32", "bf16"])
@pytest.mark.parametrize("vocab", [64, 100, 2050, 16385, 70001])
@pytest.mark.parametrize("levels", [1, 2, 40])
def test_equal_logits_come_in_the_order_of_their_tokens(lib, vocab, bf, levels):
    rng = np.random.default_rng(levels)
    z = rounded(rng.integers(0, levels, size=(4, vocab)) / 4.0, bf)
    z[1] = np.sort(z[1])                                   # the best last
    z[2] = -np.sort(-z[2])
    z[3] = np.where(z[3] == 0.0, np.where(rng.random(vocab) < 0.5, -0.0, 0.0), z[3])
    target = np.zeros(4, dtype=int)
    got = run_logprobs(lib, z, bf, target, n_top=64)
    check_logprobs(got, z, bf, target, n_top=64)


@pytest.mark.parametrize("vocab", [2048, 33333])
def test_ascending_and_descending_logits(lib, vocab):
    z = np.stack([np.arange(vocab), -np.arange(vocab), np.arange(vocab) % 2048, (np.arange(vocab) * 7919) % vocab]) * 2.0 ** -10
    target = np.full(4, vocab - 1)
    got = run_logprobs(lib, z, False, target, n_top=64, g=np.ones(4), ge=np.ones(4))
    check_logprobs(got, z, False, target, n_top=64, g=np.ones(4), ge=np.ones(4))


def test_large_logits_that_all_lie_in_the_same_places(lib):
    """In every 256 stretches of 32 tokens the same 63 have nearly all of the mass."""
    rng = np.random.default_rng(4)
    vocab = 300001
    z = rounded(rng.standard_normal((2, vocab)) * 0.5 + 10.0 * (np.arange(vocab) // 32 % 256 < 63), False)
    z[1] = rounded(np.floor(z[1] * 4) / 4, False)          # and many equal ones
    target = np.array([0, 300000])
    for n_top in (1, 63, 64):
        check_logprobs(run_logprobs(lib, z, False, target, n_top=n_top), z, False, target, n_top=n_top)


def test_any_output_may_be_left_out(lib):
    rng = np.random.default_rng(5)
    z = make_logits(rng, 3, 5000, False)
    logits, _ = place(z, False)
    desc = lib.Logits(logits)
    target = dev([1, 2, 3], np.int32)
    f = lambda *s: torch.full(s, 99.0, device=DEV)  # noqa: E731
    scratch = f(max(1, lib.pg_logprob_scratch_floats(3, 5000, 20)))
    full = dict(logp=f(3), entropy=f(3), top_logp=f(3, 20), top_ids=torch.zeros(3, 20, dtype=torch.int32, device=DEV))
    lib.pg_token_logprobs(desc, target, full["logp"], scratch, **{k: v for k, v in full.items() if k != "logp"})
    for name in full:
        one = torch.empty_like(full[name])
        lib.pg_token_logprobs(desc, target if name != "entropy" else None, one if name == "logp" else None, scratch,
                              **({name: one} if name != "logp" else {}))
        assert torch.equal(one, full[name]), name
    lib.pg_token_logprobs(desc, None, None, scratch)
    torch.cuda.synchronize()


def test_entropys_gradient_without_targets(lib):
    rng = np.random.default_rng(6)
    z = make_logits(rng, 3, 5001, True)
    logits, _ = place(z, True)
    desc = lib.Logits(logits)
    stats, d, ge = torch.empty(3, 4, device=DEV), torch.empty_like(logits), dev([1.0, -2.0, 0.5], np.float32)
    lib.pg_token_logprobs(desc, None, None, torch.empty(max(1, lib.pg_logprob_scratch_floats(3, 5001)), device=DEV), stats=stats)
    lib.pg_token_logprobs_backward(desc, None, stats, d, g_entropy=ge)
    for r in range(3):
        want = ref.token_logprobs_gradient(z[r], None, 0.0, float(ge[r]))
        s = Softmax(z[r], 1.0, None)
        coef = abs(float(ge[r])) * (abs(s.h - s.ln_s) + s.far)
        tol = s.p * (coef * (s.p_rel + 8 * U) + abs(float(ge[r])) * (s.h_tol + s.lse_tol)) + TINY
        near(d[r].double().cpu().numpy(), want, tol * (1 + 2.0 ** -7) + store_tol(want, True), f"row {r}")


@pytest.mark.parametrize("bf", [False, True], ids=["f32", "bf16"])
@pytest.mark.parametrize("rows,vocab,k", [(700, 24001, 64), (3000, 5000, 7), (150, 65537, 200), (2049, 2048, 33), (5000, 300, 256)])
def test_rows_whose_pieces_do_not_end_with_them(lib, rows, vocab, k, bf):
    """Many rows of several pieces each, shared out to workgroups: every row is right."""
    gen = torch.Generator(device=DEV).manual_seed(rows)
    z = torch.randn(rows, vocab, device=DEV, generator=gen) * 3
    z = z.to(torch.bfloat16) if bf else z
    target = torch.randint(0, vocab, (rows,), device=DEV, generator=gen).to(torch.int32)
    desc, n = lib.Logits(z), 20
    f = lambda *s: torch.full(s, 99.0, device=DEV)  # noqa: E731
    scratch = f(lib.pg_logprob_scratch_floats(rows, vocab, n))
    ln = torch.log_softmax(z.double(), 1)
    t = target.long()[:, None]
    tol = float((vocab / 256 + 64) * U + 120 * U)          # |y - top| and entropies stay below 26
    order = torch.sort(z.float(), dim=1, descending=True, stable=True)[1][:, :n]
    for top in (False, True):
        logp, entropy, stats = f(rows), f(rows), f(rows, 4)
        ids, values = torch.zeros(rows, n, dtype=torch.int32, device=DEV), f(rows, n)
        lib.pg_token_logprobs(desc, target, logp, scratch, entropy=entropy, stats=stats, **(dict(top_ids=ids, top_logp=values) if top else {}))
        assert (logp.double() - ln.gather(1, t)[:, 0]).abs().max() < tol
        assert (entropy.double() + (ln.exp() * ln).sum(1)).abs().max() < 12 * tol
        if top:
            assert torch.equal(ids.long(), order) and (values.double() - ln.gather(1, order)).abs().max() < tol
    g = torch.randn(rows, device=DEV, generator=gen)
    d = torch.empty_like(z)
    lib.pg_token_logprobs_backward(desc, target, stats, d, g_logp=g)
    want = -g.double()[:, None] * ln.exp()
    want.scatter_add_(1, t, g.double()[:, None])
    assert ((d.double() - want).abs() - want.abs() * (2.0 ** -8 if bf else U)).max() < 5 * tol
    # a list of tokens of every kind of row
    ids = torch.argsort(torch.rand(rows, vocab, device=DEV, generator=gen), dim=1)[:, :k].to(torch.int32).contiguous()
    q = torch.log_softmax(torch.randn(rows, vocab, device=DEV, generator=gen) * 3, 1).gather(1, ids.long()).contiguous()
    loss, stats = f(rows), f(rows, lib.PG_DISTILL_STATS)
    lib.pg_distill_loss(desc, ids, q, loss, scratch, tail=True, stats=stats)
    w, p = q.double().exp(), ln.exp().scatter(1, ids.long(), 0.0).sum(1)
    q_rest = (1 - w.sum(1)).clamp_min(0)
    want = (w * (q.double() - ln.gather(1, ids.long()))).sum(1)
    want += torch.where(q_rest > 0, q_rest * (q_rest.log() - p.log()), 0.0) if k < vocab else 0.0
    assert (loss.double() - want).abs().max() < 3 * tol
    lib.pg_distill_backward(desc, ids, q, stats, g, d)
    everything = (w.sum(1) + q_rest)[:, None]
    want = ln.exp() * (everything - torch.where(p > 0, q_rest / p, 0.0)[:, None])
    want.scatter_(1, ids.long(), everything * ln.exp().gather(1, ids.long()) - w)
    want *= g.double()[:, None]
    assert ((d.double() - want).abs() - want.abs() * (2.0 ** -8 if bf else U)).max() < 5 * tol


def test_more_rows_than_a_grid_has_in_one_direction(lib):
    """And short ones: every row is right, the last included."""
    rows, vocab = 70001, 11
    gen = torch.Generator(device=DEV).manual_seed(1)
    z = torch.randn(rows, vocab, device=DEV, generator=gen)
    target = torch.randint(0, vocab, (rows,), device=DEV, generator=gen).to(torch.int32)
    logp, entropy, stats = torch.empty(rows, device=DEV), torch.empty(rows, device=DEV), torch.empty(rows, 4, device=DEV)
    top_ids, top_logp = torch.empty(rows, 3, dtype=torch.int32, device=DEV), torch.empty(rows, 3, device=DEV)
    desc = lib.Logits(z)
    scratch = torch.empty(max(1, lib.pg_logprob_scratch_floats(rows, vocab, 3)), device=DEV)
    lib.pg_token_logprobs(desc, target, logp, scratch, entropy=entropy, stats=stats, top_ids=top_ids, top_logp=top_logp)
    g = torch.randn(rows, device=DEV, generator=gen)
    d = torch.empty_like(z)
    lib.pg_token_logprobs_backward(desc, target, stats, d, g_logp=g)
    zz = z.double().cpu()
    ln = torch.log_softmax(zz, 1)
    t = target.cpu().long()[:, None]
    assert (logp.cpu().double() - ln.gather(1, t)[:, 0]).abs().max() < 40 * U * 8
    assert (entropy.cpu().double() + (ln.exp() * ln).sum(1)).abs().max() < 80 * U * 8
    assert torch.equal(top_ids.cpu().long(), zz.topk(3)[1])
    want = -g.cpu().double()[:, None] * ln.exp()
    want.scatter_add_(1, t, g.cpu().double()[:, None])
    assert (d.cpu().double() - want).abs().max() < 80 * U * 6


def test_rows_that_begin_past_two_to_the_31_elements(lib):
    stride, vocab = (1 << 30) + 3, 4099
    rng = np.random.default_rng(3)
    z = make_logits(rng, 4, vocab, True)
    whole = torch.zeros(3 * stride + vocab, dtype=torch.bfloat16, device=DEV)
    view = whole.as_strided((4, vocab), (stride, 1))
    view.copy_(torch.from_numpy(z).to(DEV))
    target = np.array([0, 5, 4098, 77])
    desc, tg = lib.Logits(view), dev(target, np.int32)
    out = dict(logp=torch.empty(4, device=DEV), entropy=torch.empty(4, device=DEV), stats=torch.empty(4, 4, device=DEV),
               top_ids=torch.empty(4, 5, dtype=torch.int32, device=DEV), top_logp=torch.empty(4, 5, device=DEV))
    scratch = torch.empty(max(1, lib.pg_logprob_scratch_floats(4, vocab, 5)), device=DEV)
    lib.pg_token_logprobs(desc, tg, out["logp"], scratch, **{k: v for k, v in out.items() if k != "logp"})
    g = np.array([1.0, -1.0, 0.5, 2.0])
    lib.pg_token_logprobs_backward(desc, tg, out["stats"], view, g_logp=dev(g, np.float32))
    got = {k: v.cpu().numpy() for k, v in out.items()}
    got["d"] = view.double().cpu().numpy()
    check_logprobs(got, z, True, target, n_top=5, g=g)


# ------------------------------------------------------------------ distillation

def run_distill(lib, z, bf, ids, values, tail, g, temperature=None, open_=None, allow_row=None, stride=None, offset=0, in_place=False):
    rows, vocab = z.shape
    logits, whole = place(z, bf, stride, offset)
    more = {} if open_ is None else dict(allow=dev(mask_words(open_), np.int32), allow_row=dev(allow_row, np.int32))
    desc = lib.Logits(logits, **more)
    t = None if temperature is None else dev(temperature, np.float32)
    i, v = dev(ids, np.int32), dev(values, np.float32)
    loss, stats = torch.full((rows,), 99.0, device=DEV), torch.full((rows, lib.PG_DISTILL_STATS), 99.0, device=DEV)
    scratch = torch.full((max(1, lib.pg_distill_scratch_floats(rows, vocab)),), math.nan, device=DEV)
    lib.pg_distill_loss(desc, i, v, loss, scratch, tail=tail, temperature=t, stats=stats)
    alone = torch.full((rows,), 99.0, device=DEV)
    lib.pg_distill_loss(desc, i, v, alone, scratch, tail=tail, temperature=t)
    if in_place:
        d, d_whole = logits, whole
    else:
        d, d_whole = place(np.full(z.shape, 5.0), bf, stride, (offset + 3) % 8 if offset else 0)
    lib.pg_distill_backward(desc, i, v, stats, dev(g, np.float32), d, temperature=t)
    torch.cuda.synchronize()
    gaps = torch.ones(d_whole.shape, dtype=torch.bool, device=DEV)
    gaps.as_strided(d.shape, d.stride(), (d.data_ptr() - d_whole.data_ptr()) // d_whole.element_size()).fill_(False)
    assert (d_whole[gaps] == 7.0).all(), "something beside the rows was written"
    assert torch.equal(alone.isnan(), loss.isnan()) and torch.equal(alone.nan_to_num(), loss.nan_to_num())
    return loss.cpu().numpy(), d.double().cpu().numpy()


def check_distill(got, z, bf, ids, values, tail, g, temperature=None, open_=None, allow_row=None):
    loss, d = got
    values = np.asarray(values, dtype=np.float32).astype(np.float64)
    for r in range(len(z)):
        t = 1.0 if temperature is None else float(np.float32(temperature[r]))
        allow = None if open_ is None or allow_row[r] == -1 else open_[allow_row[r]]
        want, grad = ref.distill(z[r], ids[r], values[r], tail, t, allow)
        a = float(np.float32(g[r]))
        grad = grad * a if a != 0 else np.zeros(len(grad))
        s = Softmax(z[r], t, allow)
        tol, grad_tol = 0.0, 0.0
        if s.ok and np.isfinite(grad).all():
            seen = list(dict.fromkeys(int(i) for i in ids[r] if 0 <= i < len(z[r])))
            if seen:
                first = [list(ids[r]).index(i) for i in seen]
                v = values[r][first]
                w = np.exp(v) if tail else np.exp(v - max(v.max(), -1e300)) / max(np.sum(np.exp(v - max(v.max(), -1e300))), 1e-300)
                rest = np.ones(len(z[r]), dtype=bool)
                rest[seen] = False
                p_rest = np.sum(s.p[rest])
                q_rest = max(0.0, 1 - w.sum()) if tail and (rest & (s.p > 0)).any() else 0.0
                if np.isfinite(want):
                    tol = np.sum(w * (s.lse_tol + 4 * U * s.far[seen])) + U * abs(want)
                    if q_rest > 0:
                        tol += q_rest * (s.sum_tol + 2 * s.lse_tol + U * (4 * np.sum(s.p[rest] * s.far[rest]) / p_rest + 8)) + 1e-12
                inv = 1.0 if t == 0 else 1 / t
                everything = w.sum() + q_rest
                grad_tol = TINY + np.zeros(len(z[r]))
                if p_rest > 0:
                    share = abs(everything * p_rest - q_rest)
                    wrong = everything * p_rest * (2 * s.lse_tol + s.sum_tol + 16 * U + 4 * U * np.sum(s.p[rest] * s.far[rest]) / p_rest) + 2 * U * share
                    grad_tol = np.where(rest, s.p / p_rest * (wrong + share * (s.p_rel + s.sum_tol + 8 * U)), 0.0)
                grad_tol[seen] = everything * s.p[seen] * (s.p_rel[seen] + 8 * U) + w * U * (4 * np.abs(np.maximum(v, -1e3)) + 16)
                grad_tol = (abs(a) * inv * (grad_tol + TINY)) * (1 + 2.0 ** -7) + store_tol(grad, bf)
        near(loss[r], want, tol, f"loss of row {r}")
        near(d[r], grad, grad_tol, f"gradient of row {r}")


def teacher_lists(rng, z, k, open_=None):
    """The k most likely tokens of a distribution like the student's, with their log-probs, in falling order."""
    t = z * 0.8 + rng.standard_normal(z.shape)
    if open_ is not None:
        t = np.where(open_, t, -25.0)
    ln = t - np.log(np.exp(t - t.max(1, keepdims=True)).sum(1, keepdims=True)) - t.max(1, keepdims=True)
    ids = np.argsort(-ln, axis=1, kind="stable")[:, :k]
    return ids.astype(np.int32), np.take_along_axis(ln, ids, 1).astype(np.float32)


@pytest.mark.parametrize("tail", [False, True], ids=["top", "tail"])
@pytest.mark.parametrize("bf", [False, True], ids=["f32", "bf16"])
@pytest.mark.parametrize("rows,vocab,k", [(1, 1, 1), (3, 2, 1), (2, 9, 9), (3, 65, 20), (2, 300, 256), (2, 2049, 64), (3, 8191, 1), (2, 16384, 256), (2, 40001, 20),
                                          (1, 131073, 64)])
def test_distillation(lib, rows, vocab, k, bf, tail):
    rng = np.random.default_rng(vocab + k)
    z = make_logits(rng, rows, vocab, bf)
    ids, values = teacher_lists(rng, z, k)
    g, t = rng.standard_normal(rows), rng.uniform(0.6, 1.5, size=rows)
    for place_as in ({}, dict(stride=vocab + 3, offset=1), dict(in_place=True)):
        check_distill(run_distill(lib, z, bf, ids, values, tail, g, t, **place_as), z, bf, ids, values, tail, g, t)


@pytest.mark.parametrize("tail", [False, True], ids=["top", "tail"])
@pytest.mark.parametrize("bf", [False, True], ids=["f32", "bf16"])
@pytest.mark.parametrize("vocab,k", [(40, 6), (3001, 40), (20000, 200)])
def test_distillations_lists(lib, vocab, k, bf, tail):
    """Duplicates, tokens that do not exist, empty lists, values of -inf, shifted ones, masks, a weight of 0."""
    rng = np.random.default_rng(k)
    rows = 16
    z = make_logits(rng, rows, vocab, bf)
    open_ = np.stack([rng.random(vocab) < 0.7, np.zeros(vocab, dtype=bool)])
    open_[0, 0] = True
    allow_row = np.full(rows, -1)
    allow_row[[3, 4, 5]] = 0
    allow_row[6] = 1
    ids, values = teacher_lists(rng, z, k, np.where((allow_row == 0)[:, None], open_[0], True))
    ids[0, k // 2:] = ids[0, 0]                            # the first of equal ids counts
    ids[1, 1:4], values[1, 1:4] = [-1, vocab, -7], np.nan  # passed over, whatever their values are
    ids[2] = -1                                            # no list
    ids[4, 2] = np.flatnonzero(~open_[0])[0]               # a token that is not allowed: loss +inf
    values[5, 0] = -np.inf                                 # listed, with nothing
    values[7] = -np.inf                                    # all of the mass is elsewhere, or nowhere
    values[8] = values[8] + 5.0                            # more mass than there is
    ids[9] = rng.permutation(ids[9])
    values[10, k - 1] = np.nan
    values[11, k - 1] = np.inf
    values[12] -= 30.0                                     # hardly any mass listed
    z[13, ids[13, 0]] = -np.inf                            # the student has none there: +inf
    z[14, :] = rounded(z[14] - 20000.0, bf)
    z[15, vocab // 2] = np.nan
    g = rng.standard_normal(rows)
    g[9] = 0.0
    got = run_distill(lib, z, bf, ids, values, tail, g, None, open_, allow_row)
    check_distill(got, z, bf, ids, values, tail, g, None, open_, allow_row)
    assert got[0][2] == 0 and got[0][6] == 0 and np.isinf(got[0][4]) and np.isinf(got[0][13]) and np.isnan(got[0][[10, 11, 15]]).all()


def test_a_workgroups_part_of_a_row_that_has_more_bits_than_lds(lib):
    """1400 rows of 200001 tokens: a workgroup's share is 67 stretches, and 64 of them have their bits at a time."""
    rows, vocab, k = 1400, 200001, 256
    gen = torch.Generator(device=DEV).manual_seed(2)
    z = torch.randn(rows, vocab, device=DEV, generator=gen).mul_(3).to(torch.bfloat16)
    ids = torch.randint(0, vocab, (rows, k), device=DEV, generator=gen).to(torch.int32)
    values = torch.log_softmax(torch.randn(rows, k + 1, device=DEV, generator=gen), 1)[:, :k].contiguous()
    desc = lib.Logits(z)
    loss, stats = torch.empty(rows, device=DEV), torch.empty(rows, lib.PG_DISTILL_STATS, device=DEV)
    lib.pg_distill_loss(desc, ids, values, loss, torch.empty(lib.pg_distill_scratch_floats(rows, vocab), device=DEV), tail=True, stats=stats)
    g = torch.randn(rows, device=DEV, generator=gen)
    some = [0, 1, 2, 699, 700, 1398, 1399]
    before = z[some].double().cpu().numpy()
    lib.pg_distill_backward(desc, ids, values, stats, g, z)
    pick = lambda t: t[some].cpu().numpy()  # noqa: E731
    check_distill((pick(loss), z[some].double().cpu().numpy()), before, True, pick(ids), pick(values), True, pick(g))


@pytest.mark.parametrize("vocab", [50, 5000])
def test_a_tail_that_hardly_exists(lib, vocab):
    """The listed tokens have nearly all of the mass, the student's or the teacher's: what is left is not lost in a difference."""
    rng = np.random.default_rng(11)
    z = make_logits(rng, 4, vocab, False, 1.0)
    ids = np.argsort(-z, axis=1)[:, :20].astype(np.int32)
    for r, up in enumerate((0.0, 20.0, 40.0, 80.0)):
        np.put_along_axis(z[r:r + 1], ids[r:r + 1], np.take_along_axis(z[r:r + 1], ids[r:r + 1], 1) + up, 1)
    z = rounded(z, False)
    values = np.log(np.full((4, 20), (1 - np.array([0.5, 1e-6, 1e-3, 1e-2]))[:, None] / 20))
    g = np.ones(4)
    for tail in (False, True):
        check_distill(run_distill(lib, z, False, ids, values, tail, g), z, False, ids, values, tail, g)


# ------------------------------------------------------------------ the clipped objective

def run_surrogate(lib, seqs, lo, hi, refs=None, kl_coef=0.0, weight=None, max_len=None, alias=False, slack=3):
    """seqs: [(logp, old, adv)]; slack: tokens behind the last sequence."""
    lens = [len(s[0]) for s in seqs]
    cu = np.cumsum([0] + lens)
    n = int(cu[-1]) + slack
    flat = lambda parts: dev(np.concatenate([np.asarray(p, dtype=np.float32) for p in parts] + [np.full(slack, 7.0, dtype=np.float32)]), np.float32)  # noqa: E731
    logp, old = flat([s[0] for s in seqs]), flat([s[1] for s in seqs])
    most = max(lens + [1]) if max_len is None else max_len
    f = lambda m: torch.full((m,), 99.0, device=DEV)  # noqa: E731
    out = dict(objective=f(len(seqs)), kl=f(len(seqs)), clipped=torch.full((len(seqs),), 99, dtype=torch.int32, device=DEV),
               g_logp=logp if alias else torch.full((n,), 7.0, device=DEV))
    need = lib.pg_surrogate_scratch_floats(len(seqs), most)
    lib.pg_token_surrogate(logp, old, dev([s[2] for s in seqs], np.float32), dev(cu, np.int32), out["objective"], out["g_logp"], lo, hi, most,
                           torch.full((need,), math.nan, device=DEV) if need else None, logp_ref=None if refs is None else flat(refs), kl_coef=kl_coef,
                           weight=None if weight is None else dev(weight, np.float32), kl=out["kl"], clipped=out["clipped"])
    torch.cuda.synchronize()
    got = {k: v.cpu().numpy() for k, v in out.items()}
    assert (got["g_logp"][n - slack:] == 7.0).all(), "tokens behind the last sequence were written"
    return got


def check_surrogate(got, seqs, lo, hi, refs=None, kl_coef=0.0, weight=None):
    at = 0
    f32 = lambda x: np.asarray(x, dtype=np.float32).astype(np.float64)  # noqa: E731
    kl_coef = float(np.float32(kl_coef))
    for r, (logp, old, adv) in enumerate(seqs):
        logp, old, adv = f32(logp), f32(old), float(f32(adv))
        w = None if weight is None else float(f32(weight[r]))
        x = None if refs is None else f32(refs[r])
        want = ref.surrogate(logp, old, adv, lo, hi, x, kl_coef, w)
        n = len(logp)
        g = got["g_logp"][at:at + n]
        at += n
        if n == 0:
            assert got["objective"][r] == 0 and got["kl"][r] == 0 and got["clipped"][r] == 0
            continue
        assert got["clipped"][r] == want["clipped"], f"cut tokens of sequence {r}"
        w = 1 / n if w is None else w
        with np.errstate(over="ignore", invalid="ignore"):
            d = logp - old
            ra = np.abs(np.exp(d) * adv) if adv else np.zeros(n)
            term_tol = ra * U * (np.abs(d) + 8)
            g_tol = term_tol.copy()
            k_tol = np.zeros(n)
            if x is not None:
                # k is a series for small x and a difference of numbers of at most e^x + |x| + 1 elsewhere
                e, k = np.expm1(x - logp), np.expm1(x - logp) - (x - logp)
                k_tol = U * (16 * k + np.where(np.abs(x - logp) > 0.4, 4 * (e + 2 + np.abs(x - logp)) + 2 * np.abs(x - logp) * (e + 1), 0.0))
                g_tol = g_tol + abs(kl_coef) * U * (np.abs(e) * 16 + np.abs(x - logp) * (e + 1) * 4)
            size = np.nan_to_num(np.minimum(ra, (1 + min(hi, 1e30)) * abs(adv)), posinf=0)
            tol = w * np.sum(np.nan_to_num(term_tol) + abs(kl_coef) * k_tol + 40 * U * size) + 40 * U * abs(want["objective"]) + 2.0 ** -147      # below 2^-126 numbers are multiples of 2^-149
            mean = np.mean(k_tol) + 40 * U * want["kl"]
            g_tol = abs(w) * g_tol + 4 * U * np.abs(want["g_logp"]) + 1e-37
        near(got["objective"][r], want["objective"], tol, f"objective of sequence {r}")
        near(got["kl"][r], want["kl"], mean, f"divergence of sequence {r}")
        near(g, want["g_logp"], g_tol, f"gradient of sequence {r}")


def some_sequences(rng, lens, spread=0.25):
    out = []
    for n in lens:
        logp = -np.abs(rng.standard_normal(n)) * 2
        out.append((logp, logp + rng.standard_normal(n) * spread, float(rng.standard_normal())))
    return out


@pytest.mark.parametrize("lens", [[1], [0, 1, 2, 0], [3, 0, 64, 65, 255, 256, 257], [1023, 1024, 1025, 4096, 1], [20000, 3, 0, 4097, 8191, 8192, 8193], [131071], [1] * 700])
def test_surrogate(lib, lens):
    rng = np.random.default_rng(sum(lens))
    seqs = some_sequences(rng, lens)
    refs = [np.asarray(s[0]) + rng.standard_normal(len(s[0])) * 0.5 for s in seqs]
    weight = rng.uniform(0.1, 2.0, size=len(lens))
    for more in (dict(), dict(refs=refs, kl_coef=0.04), dict(weight=weight), dict(refs=refs, kl_coef=0.3, weight=weight)):
        check_surrogate(run_surrogate(lib, seqs, 0.2, 0.28, **more), seqs, 0.2, 0.28, **more)
    for lo, hi in ((0.0, 0.0), (1.0, math.inf)):
        check_surrogate(run_surrogate(lib, seqs, lo, hi, alias=True), seqs, lo, hi)
    # a length that is not the largest sizes the split alone
    for most in (0, 1, max(lens) // 2, max(lens) * 3):
        check_surrogate(run_surrogate(lib, seqs, 0.2, 0.2, refs=refs, kl_coef=0.1, max_len=most), seqs, 0.2, 0.2, refs=refs, kl_coef=0.1)


def test_surrogate_far_off_policy_and_without_numbers(lib):
    inf = math.inf
    seqs = [([-1.0, -2.0, -3.0], [-200.0, -2.0, -3.0], 0.0),           # an infinite ratio without an advantage
            ([-1.0, -2.0], [-60.0, -90.0], 1.0), ([-1.0, -2.0], [-60.0, -50.0], -1.0),
            ([-inf, -1.0], [-1.0, -1.0], 1.0), ([-inf, -1.0], [-1.0, -1.0], -1.0),
            ([math.nan, -1.0], [-1.0, -1.0], 1.0), ([-1.0, -1.0], [-1.0, -1.0], math.nan), ([-1.0], [-1.5], 1e-30), ([-100.0], [-1.0], 1.0)]
    check_surrogate(run_surrogate(lib, seqs, 0.2, 0.2), seqs, 0.2, 0.2)
    seqs, refs = [seqs[i] for i in (0, 1, 2, 5, 7)], [[-1.0, -2.0, -3.0], [-1e-4 - 1.0, -2.0 + 1e-6], [-30.0, -1.0], [-1.0, -1.0], [-1.0]]
    check_surrogate(run_surrogate(lib, seqs, 0.2, 0.2, refs=refs, kl_coef=0.1), seqs, 0.2, 0.2, refs=refs, kl_coef=0.1)


def test_surrogate_reads_nothing_past_bad_offsets(lib):
    """Offsets are cut to the tokens there are, and a sequence that would end before it begins is empty."""
    n = 50
    logp = torch.full((n,), -1.0, device=DEV)
    g, objective = torch.full((n,), 7.0, device=DEV), torch.full((4,), 99.0, device=DEV)
    clipped = torch.full((4,), 99, dtype=torch.int32, device=DEV)
    lib.pg_token_surrogate(logp, logp.clone(), torch.ones(4, device=DEV), dev([-20, 10, 5, 1 << 30, 2000000000], np.int32), objective, g, 0.2, 0.2, 100,
                           torch.empty(max(1, lib.pg_surrogate_scratch_floats(4, 100)), device=DEV), clipped=clipped)
    assert objective.tolist() == [1.0, 0.0, 1.0, 0.0] and clipped.tolist() == [0] * 4
    assert (g != 7.0).all()


# ------------------------------------------------------------------ together

def chain(lib, s):
    lib.pg_token_logprobs(s["desc"], s["target"], s["logp"], s["scratch"], temperature=s["t"], entropy=s["entropy"], stats=s["stats"])
    lib.pg_token_surrogate(s["logp"], s["old"], s["adv"], s["cu"], s["objective"], s["g"], 0.2, 0.28, 16, s["more"], logp_ref=s["ref"], kl_coef=0.05)
    lib.pg_token_logprobs_backward(s["desc"], s["target"], s["stats"], s["d"], g_logp=s["g"], g_entropy=s["ge"], temperature=s["t"])


def chain_state(lib, seed=0, rows=40, vocab=9001):
    rng = np.random.default_rng(seed)
    z = make_logits(rng, rows, vocab, False)
    logits, _ = place(z, False)
    target = rng.integers(0, vocab, size=rows)
    t = rng.uniform(0.7, 1.3, size=rows)
    logp = np.array([ref.token_logprobs(z[r], target[r], float(np.float32(t[r])))["logp"] for r in range(rows)])
    f = lambda *n: torch.empty(*n, device=DEV)  # noqa: E731
    lens = [16, 1, 0, 15, 8]
    s = dict(z=z, logits=logits, desc=lib.Logits(logits), target=dev(target, np.int32), t=dev(t, np.float32), logp=f(rows), entropy=f(rows), stats=f(rows, 4),
             scratch=f(max(1, lib.pg_logprob_scratch_floats(rows, vocab))), more=f(max(1, lib.pg_surrogate_scratch_floats(5, 16))),
             old=dev(logp + rng.standard_normal(rows) * 0.1, np.float32), ref=dev(logp + rng.standard_normal(rows) * 0.2, np.float32),
             adv=dev(rng.standard_normal(5), np.float32), cu=dev(np.cumsum([0] + lens), np.int32), objective=f(5), g=f(rows), d=torch.empty_like(logits),
             ge=torch.full((rows,), 0.01, device=DEV), lens=lens)
    return s


def objective_of(s, z):
    """The whole objective in fp64: sum of the sequences' and 0.01 of the entropies."""
    at, total = 0, 0.0
    old, x, adv, t, target = (s[k].double().cpu().numpy() for k in ("old", "ref", "adv", "t", "target"))
    rows = [ref.token_logprobs(z[r], int(target[r]), t[r]) for r in range(len(z))]
    for r, n in enumerate(s["lens"]):
        logp = np.array([q["logp"] for q in rows[at:at + n]])
        total += ref.surrogate(logp, old[at:at + n], adv[r], 0.2, 0.28, x[at:at + n], float(np.float32(0.05)))["objective"]
        at += n
    return total + float(np.float32(0.01)) * sum(q["entropy"] for q in rows)


def test_a_step_of_the_policy_against_differences(lib):
    s = chain_state(lib)
    chain(lib, s)
    d = s["d"].double().cpu().numpy()
    assert abs(float(s["objective"].sum()) + 0.01 * float(s["entropy"].sum()) - objective_of(s, s["z"])) < 1e-4
    rng = np.random.default_rng(1)
    target = s["target"].cpu().numpy()
    for _ in range(4):
        way = rng.standard_normal(s["z"].shape) * 0.01
        way[np.arange(len(way)), target] += rng.standard_normal(len(way))          # along what the log-probs feel
        h = 1e-6
        slope = (objective_of(s, s["z"] + h * way) - objective_of(s, s["z"] - h * way)) / (2 * h)
        # fp32 gradients of 40 x 9001 logits: 1e-5 of the sum of what is multiplied; differences: h^2 and 1e-15 / h of the objective
        assert abs(slope - np.sum(d * way)) < 1e-5 * np.sum(np.abs(d * way)) + 1e-7


def test_a_captured_step_replays_as_the_eager_one(lib):
    s = chain_state(lib, 2)
    names = ("logp", "entropy", "objective", "g", "d")
    chain(lib, s)
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        chain(lib, s)
    for k in range(4):
        s["logits"].copy_(torch.randn(s["logits"].shape, device=DEV, generator=torch.Generator(device=DEV).manual_seed(k)) * 3)
        graph.replay()
        torch.cuda.synchronize()
        replayed = {n: s[n].clone() for n in names}
        for n in names:
            s[n].fill_(99.0)
        chain(lib, s)                                      # and the program's own eager work between the replays
        torch.cuda.synchronize()
        for n in names:
            assert torch.equal(replayed[n], s[n]), (k, n)


def test_calls_on_two_streams_at_once(lib):
    states = [chain_state(lib, 5), chain_state(lib, 6)]
    names = ("logp", "entropy", "objective", "g", "d")
    want = []
    for s in states:
        chain(lib, s)
        torch.cuda.synchronize()
        want.append({n: s[n].clone() for n in names})
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(5):
        for s, stream in zip(states, streams):
            with torch.cuda.stream(stream):
                chain(lib, s)
    torch.cuda.synchronize()
    for s, w in zip(states, want):
        for n in names:
            assert torch.equal(s[n], w[n]), n


def test_the_teachers_alternatives_are_a_list_to_learn_from(lib):
    """A student that is the teacher has nothing to learn; another has, with the slope that the gradient says."""
    rng = np.random.default_rng(9)
    rows, vocab, k = 12, 5003, 64
    teacher, _ = place(make_logits(rng, rows, vocab, False), False)
    ids, values = torch.empty(rows, k, dtype=torch.int32, device=DEV), torch.empty(rows, k, device=DEV)
    t = torch.full((rows,), 1.3, device=DEV)
    lib.pg_token_logprobs(lib.Logits(teacher), None, None, torch.empty(max(1, lib.pg_logprob_scratch_floats(rows, vocab, k)), device=DEV), temperature=t,
                          top_ids=ids, top_logp=values)
    scratch = torch.empty(max(1, lib.pg_distill_scratch_floats(rows, vocab)), device=DEV)
    loss, stats, d = torch.empty(rows, device=DEV), torch.empty(rows, lib.PG_DISTILL_STATS, device=DEV), torch.empty_like(teacher)
    one = torch.ones(rows, device=DEV)

    def learn(logits, tail):
        desc = lib.Logits(logits)
        lib.pg_distill_loss(desc, ids, values, loss, scratch, tail=tail, temperature=t, stats=stats)
        lib.pg_distill_backward(desc, ids, values, stats, one, d, temperature=t)
        return float(loss.sum())

    assert abs(learn(teacher, True)) < rows * 5e-5 and float(d.abs().max()) < 1e-5
    student, _ = place(make_logits(rng, rows, vocab, False), False)
    way = torch.randn(student.shape, device=DEV, generator=torch.Generator(device=DEV).manual_seed(3))
    for tail in (False, True):
        slope = (learn(student + 0.01 * way, tail) - learn(student - 0.01 * way, tail)) / 0.02
        assert learn(student, tail) > 1.0
        # differences: third derivatives of a few units times 0.01^2, and the rounding of losses of about ten over 0.02
        want = float((d.double() * way).sum())
        assert abs(slope - want) < 1e-2 * (1 + abs(want)), (slope, want)


def test_results_do_not_change_from_run_to_run(lib):
    rng = np.random.default_rng(12)
    z = make_logits(rng, 7, 50001, True)
    ids, values = teacher_lists(rng, z, 100)
    target = rng.integers(0, 50001, size=7)
    g = rng.standard_normal(7)
    a = run_logprobs(lib, z, True, target, n_top=64, g=g, ge=g)
    x = run_distill(lib, z, True, ids, values, True, g)
    for _ in range(4):
        b = run_logprobs(lib, z, True, target, n_top=64, g=g, ge=g)
        assert all(np.array_equal(a[k], b[k]) for k in a)
        y = run_distill(lib, z, True, ids, values, True, g)
        assert np.array_equal(x[0], y[0]) and np.array_equal(x[1], y[1])
