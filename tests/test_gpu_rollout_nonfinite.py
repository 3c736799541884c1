"""NaN and infinities inside a row's length: attention gives what the softmax gives, wherever the work is split."""
import math

import numpy as np
import pytest
import torch

from oracle import rollout as ref
from test_gpu_rollout import DEV, U24, bf16, dev, make_cache, say

pytestmark = pytest.mark.gpu
KV, HEADS = 2, 6
# rows of one call that are one workgroup each, and of one that is cut into ranges, some of which hold the last token alone
SHORT, LONG = [1, 33, 200, 0, 130], [1, 5000, 33, 0, 9001]


class Case:
    def __init__(self, lib, lens, hd, page, f8, seed):
        self.lib, self.lens, self.hd, self.page, self.f8 = lib, lens, hd, page, f8
        self.rng = np.random.default_rng([seed, hd, page, f8])
        self.cache, self.table, self.rows = make_cache(lib, self.rng, lens, KV, hd, page, f8)
        self.q = bf16(self.rng.standard_normal((len(lens), HEADS, hd))).float().numpy()

    def put(self, what, r, token, channel, value):
        """A key (0) or value (1) of row r, of the last key/value head."""
        p, slot, h = int(self.table[r, token // self.page]), token % self.page, KV - 1
        x = torch.tensor(0x7F, dtype=torch.uint8) if self.f8 else torch.tensor(value, dtype=torch.bfloat16)
        (self.cache.k[-1, p, h, slot] if what == 0 else self.cache.v[-1, p, h, :, slot])[channel] = x.to(DEV)
        self.rows[r][what][h, token, channel] = value

    def check(self, ranges, empty=()):
        """Against 64 bits; `empty`: (row, head) whose scores are all -inf."""
        n = len(self.lens)
        q, lens = bf16(self.q).to(DEV), dev(self.lens)
        out, lse = torch.zeros(n, HEADS, self.hd, dtype=torch.bfloat16, device=DEV), torch.zeros(n, HEADS, device=DEV)
        size = self.lib.pg_paged_attention_workspace(self.cache, n, HEADS, max(self.lens))
        assert not ranges or size > 0
        # floats of what an earlier call may have left
        ws = torch.full((max(16, size) // 4 + 1,), math.nan, device=DEV)
        self.lib.pg_paged_attention(self.cache, 0, q, self.table, lens, out, max(self.lens), ws, lse=lse)
        self.lib.pg_cache_check(self.cache)
        got, got_lse, asked = out.float().cpu().numpy(), lse.cpu().numpy(), q.float().cpu().numpy()
        for r, m in enumerate(self.lens):
            k, v = self.rows[r]
            with np.errstate(invalid="ignore"):
                want, want_lse, _ = ref.attention(asked[r].astype(np.float64), k, v, 1 / math.sqrt(self.hd))
            for h in range(HEADS):
                if (r, h) in empty:
                    want[h], want_lse[h] = 0.0, -math.inf
            fine = lambda a: np.where(np.isfinite(a), np.abs(a), 0.0)  # noqa: E731
            # as for finite rows: scores summed in fp32, probabilities kept to 17 bits
            far = 4 * self.hd * U24 * max(1.0, float((fine(k).max(initial=0) * fine(asked[r]).sum(1).max()) / math.sqrt(self.hd)))
            tol = (2.0 ** -15 + 2 * far) * fine(v).max(initial=0.0)
            np.testing.assert_array_equal(np.isnan(got[r]), np.isnan(want), err_msg=f"NaN of row {r}")
            lo, hi = (torch.from_numpy(b).to(torch.bfloat16).float().numpy() for b in (want - tol, want + tol))
            assert (np.isnan(want) | ((lo <= got[r]) & (got[r] <= hi))).all(), r
            np.testing.assert_array_equal(np.isnan(got_lse[r]), np.isnan(want_lse), err_msg=f"NaN of row {r}'s lse")
            ok = np.isfinite(want_lse)
            assert (np.abs(got_lse[r][ok] - want_lse[ok]) <= far + 8 * U24 * (np.abs(want_lse[ok]) + 1)).all(), r
            assert (got_lse[r] == want_lse)[~ok & ~np.isnan(want_lse)].all(), r


FORMS = [(SHORT, 64, 16, False, False), (SHORT, 128, 64, True, False), (SHORT, 32, 128, False, False), (LONG, 128, 64, False, True), (LONG, 64, 16, True, True)]


@pytest.mark.parametrize("lens,hd,page,f8,ranges", FORMS)
def test_a_query_of_nan_gives_nan(lib, lens, hd, page, f8, ranges):
    say(f"NaN query, rows {lens}, head width {hd}")
    c = Case(lib, lens, hd, page, f8, 1)
    c.q[:, 1] = math.nan
    c.q[2, 4, 7] = math.nan
    c.check(ranges)


@pytest.mark.parametrize("lens,hd,page,f8,ranges", FORMS)
def test_a_key_of_nan_gives_nan_wherever_it_lies(lib, lens, hd, page, f8, ranges):
    """The only key of its row; the last of a row, alone in its wave or step; one among many."""
    say(f"NaN keys, rows {lens}, head width {hd}")
    for at in (lambda n: n - 1, lambda n: n // 2, lambda n: 0):
        c = Case(lib, lens, hd, page, f8, 2)
        for r, n in enumerate(lens):
            if n:
                c.put(0, r, at(n), 3, math.nan)
        c.check(ranges)


@pytest.mark.parametrize("lens,hd,page,f8,ranges", FORMS)
def test_a_value_of_nan_stays_in_its_channel(lib, lens, hd, page, f8, ranges):
    say(f"NaN values, rows {lens}, head width {hd}")
    c = Case(lib, lens, hd, page, f8, 3)
    for r, n in enumerate(lens):
        if n:
            c.put(1, r, n - 1, 5, math.nan)
    c.check(ranges)


@pytest.mark.parametrize("lens,hd,page,f8,ranges", [f for f in FORMS if not f[3]])
def test_scores_of_minus_infinity_have_no_weight(lib, lens, hd, page, f8, ranges):
    """Keys whose scores are -inf fill a wave's first step, a whole piece of the row, or all of it."""
    say(f"scores of -inf, rows {lens}, head width {hd}")
    for first, last in ((lambda n: 0, lambda n: min(n - 1, 32)), (lambda n: 0, lambda n: n - 1), (lambda n: n - min(n - 1, 40), lambda n: n),
                        (lambda n: 0, lambda n: n)):
        c = Case(lib, lens, hd, page, f8, 4)
        c.q[:, :, 2] = np.abs(c.q[:, :, 2]) + 1
        for r, n in enumerate(lens):
            for t in range(first(n), max(last(n), 0)):
                c.rows[r][0][KV - 1, t, 2] = -math.inf
                c.cache.k[-1, int(c.table[r, t // page]), KV - 1, t % page, 2] = -math.inf
        whole = last(5) == 5 and first(5) == 0
        c.check(ranges, empty=[(r, h) for r, n in enumerate(lens) for h in range(HEADS // KV * (KV - 1), HEADS) if whole and n])


def test_a_score_of_plus_infinity_gives_nan(lib):
    c = Case(lib, SHORT, 64, 16, False, 5)
    c.q[:, :, 2] = 1.0
    c.put(0, 2, 150, 2, math.inf)
    c.check(False)


@pytest.mark.parametrize("lens,hd,page,f8,ranges", [f for f in FORMS if not f[3]])
def test_an_infinite_value_is_an_infinite_output(lib, lens, hd, page, f8, ranges):
    """Of the only token, whose probability is 1, of the last and of one in the middle; in its channel alone."""
    say(f"infinite values, rows {lens}, head width {hd}")
    for value, at in ((math.inf, lambda n: n - 1), (-math.inf, lambda n: n // 2), (math.inf, lambda n: 0)):
        c = Case(lib, lens, hd, page, f8, 6)
        for r, n in enumerate(lens):
            if n:
                c.put(1, r, at(n), 9, value)
        c.check(ranges)
