"""CPU-only checks of what a token policy learns from: refusals on the host before any launch, sizes, and pins of the fp64 oracle."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

from oracle import token_loss as ref
from paper_2512_15347_amd import binding as pg

P = 1 << 20                                              # an address that nothing reads: calls are refused before a launch
F = pg._lib


def logits(**change):
    d = pg.pg_logits(logits=P, stride=100, dtype=0, rows=3, vocab=100)
    for n, v in change.items():
        setattr(d, n, v)
    return C.byref(d)


FAR = 1 << 30


def forward(d, target=FAR, logp=FAR, stats=FAR, n_top=0, ids=None, top=None, scratch=FAR):
    return F.pg_token_logprobs(d, None, target, logp, FAR, stats, n_top, ids, top, scratch, None)


def backward(d, target=FAR, stats=FAR, g=FAR, ge=None, out=FAR, stride=100):
    return F.pg_token_logprobs_backward(d, None, target, stats, g, ge, out, stride, None)


def distill(d, mode=0, ids=FAR, values=FAR, k=5, loss=FAR, stats=FAR, scratch=FAR):
    return F.pg_distill_loss(d, None, mode, ids, values, k, loss, stats, scratch, None)


def distill_back(d, ids=FAR, values=FAR, k=5, stats=FAR, g=FAR, out=FAR, stride=100):
    return F.pg_distill_backward(d, None, ids, values, k, stats, g, out, stride, None)


@pytest.mark.parametrize("change,status", [
    (dict(rows=-1), pg.PG_EINVAL), (dict(vocab=0), pg.PG_EINVAL), (dict(dtype=2), pg.PG_EINVAL), (dict(logits=None), pg.PG_EINVAL),
    (dict(stride=99), pg.PG_EINVAL), (dict(logits=P + 2), pg.PG_ESHAPE), (dict(dtype=1, logits=P + 1), pg.PG_ESHAPE),
    (dict(tokens=P, n_tokens=P, tokens_stride=4, repetition=P), pg.PG_EINVAL), (dict(tokens=P, n_tokens=P, tokens_stride=4), pg.PG_EINVAL),
    (dict(bias_offsets=P, n_bias=2, bias_ids=P, bias_values=P), pg.PG_EINVAL), (dict(bias_offsets=P), pg.PG_EINVAL),
    (dict(allow=P), pg.PG_EINVAL), (dict(allow=P, n_masks=2), pg.PG_EINVAL), (dict(vocab=(1 << 30) + 1, stride=1 << 31), pg.PG_ESHAPE),
    (dict(rows=(1 << 23) + 1), pg.PG_ESHAPE), (dict(rows=1 << 22, vocab=1 << 20, stride=1 << 20), pg.PG_ESHAPE)])
def test_bad_logits_are_refused(change, status):
    d = logits(**change)
    assert [forward(d), backward(d), distill(d), distill_back(d)] == [status] * 4
    assert len(pg.pg_last_error()) > 10


def test_none_and_no_rows():
    for call in (forward, backward, distill, distill_back):
        assert call(None) == pg.PG_EINVAL
        assert call(logits(rows=0, logits=None)) == pg.PG_OK


def test_logprobs_refuse_bad_arguments():
    d = logits()
    assert forward(d, n_top=-1) == pg.PG_EINVAL and forward(d, n_top=pg.PG_TOP_MAX + 1) == pg.PG_ESHAPE
    assert forward(d, target=None) == pg.PG_EINVAL                                  # log-probs of what?
    assert forward(d, stats=FAR + 8) == pg.PG_ESHAPE
    assert backward(d, stats=None) == pg.PG_EINVAL and backward(d, stats=FAR + 4) == pg.PG_ESHAPE
    assert backward(d, target=None) == pg.PG_EINVAL
    assert backward(d, out=None) == pg.PG_EINVAL and backward(d, out=FAR + 2) == pg.PG_ESHAPE and backward(d, stride=99) == pg.PG_ESHAPE
    assert backward(logits(dtype=1), out=FAR + 1) == pg.PG_ESHAPE


def test_scratch_is_wanted_where_it_is_needed():
    d = logits(vocab=100000, stride=100000)
    if pg.pg_logprob_scratch_floats(3, 100000, 20):
        assert forward(d, n_top=20, ids=FAR, scratch=None) == pg.PG_EINVAL
        assert forward(d, n_top=20, ids=FAR, scratch=FAR + 4) == pg.PG_ESHAPE
    if pg.pg_distill_scratch_floats(3, 100000):
        assert distill(d, scratch=None) == pg.PG_EINVAL
        assert distill(d, scratch=FAR + 4) == pg.PG_ESHAPE


@pytest.mark.parametrize("call", [backward, distill_back])
@pytest.mark.parametrize("dtype,stride,out,out_stride", [
    (0, 100, P, 101), (1, 100, P, 104), (0, 100, P + 4, 100), (0, 100, P - 4, 100), (0, 100, P + 4 * 299, 100), (1, 100, P - 2 * 99, 100),
    (0, 250, P + 4 * 99, 250), (0, 100, P + 4 * 40, 300), (1, 400, P + 2 * 99, 200)])
def test_gradients_that_overlap_the_logits_are_refused(call, dtype, stride, out, out_stride):
    assert call(logits(dtype=dtype, stride=stride), out=out, stride=out_stride) == pg.PG_EINVAL
    assert "overlap" in pg.pg_last_error()


def test_distillation_refuses_bad_arguments():
    d = logits()
    assert distill(d, mode=2) == pg.PG_EINVAL and distill(d, mode=-1) == pg.PG_EINVAL
    for call in (distill, distill_back):
        assert call(d, k=0) == pg.PG_EINVAL and call(d, k=pg.PG_DISTILL_MAX + 1) == pg.PG_ESHAPE
        assert call(d, ids=None) == pg.PG_EINVAL and call(d, values=None) == pg.PG_EINVAL
        assert call(d, stats=FAR + 8) == pg.PG_ESHAPE
    assert distill(d, loss=None) == pg.PG_EINVAL
    assert distill_back(d, stats=None) == pg.PG_EINVAL and distill_back(d, g=None) == pg.PG_EINVAL
    assert distill_back(d, out=None) == pg.PG_EINVAL and distill_back(d, stride=99) == pg.PG_ESHAPE


def surrogate(logp=P, old=P, adv=P, cu=P, n=3, tokens=10, most=5, lo=0.2, hi=0.2, beta=0.0, scratch=P):
    return F.pg_token_surrogate(logp, old, None, adv, None, cu, n, tokens, most, lo, hi, beta, P, None, None, P, scratch, None)


def test_the_objective_refuses_bad_arguments():
    for change in (dict(n=-1), dict(tokens=-1), dict(most=-1), dict(lo=-0.1), dict(lo=1.1), dict(lo=math.nan), dict(hi=-0.1), dict(hi=math.nan),
                   dict(beta=math.nan), dict(beta=math.inf), dict(logp=None), dict(old=None), dict(adv=None), dict(cu=None)):
        assert surrogate(**change) == pg.PG_EINVAL, change
    assert surrogate(n=(1 << 23) + 1) == pg.PG_ESHAPE
    assert surrogate(n=0, adv=None, cu=None) == pg.PG_OK
    if pg.pg_surrogate_scratch_floats(3, 1 << 20):
        assert surrogate(most=1 << 20, scratch=None) == pg.PG_EINVAL


def test_a_coefficient_past_fp32s_range_is_refused():
    """The kernels take it in fp32, where it would be infinite and 0 times it no number."""
    for beta in (1e39, -1e300):
        assert surrogate(beta=beta) == pg.PG_EINVAL, beta
    assert surrogate(n=0, beta=3e38) == pg.PG_OK


# ---------------------------------------------------------------- sizes that are asked for once hold for smaller calls

ROWS = sorted({1, 2, 3, 7, 48, 640, 700, 2049, 65535, 65536, 1 << 20} | set(range(5, 3000, 61)) | {b + i for b in (256, 512, 1280, 2048, 4096) for i in (-1, 0, 1)})
VOCABS = [1, 17, 2047, 2048, 2049, 4097, 8191, 8193, 16384, 16385, 32001, 65537, 131073, 1 << 20, 1 << 23]


@pytest.mark.parametrize("n_top", [0, 1, 64])
def test_scratch_does_not_shrink(n_top):
    for size in (lambda r, v: pg.pg_logprob_scratch_floats(r, v, n_top), pg.pg_distill_scratch_floats):
        for v in VOCABS:
            sizes = [size(r, v) for r in ROWS]
            assert sizes == sorted(sizes), v
        for r in ROWS:
            sizes = [size(r, v) for v in VOCABS]
            assert sizes == sorted(sizes), r
        assert size(0, 5) == 0 and size(5, 0) == 0
    for r, v in ((3, 100), (48, 16384), (4096, 131073)):
        sizes = [pg.pg_logprob_scratch_floats(r, v, n) for n in (0, 1, 2, 20, 63, 64)]
        assert sizes == sorted(sizes)
    for n in (1, 3, 700, 100000):
        sizes = [pg.pg_surrogate_scratch_floats(n, m) for m in (0, 1, 100, 4096, 4097, 8192, 8193, 131071, 1 << 30)]
        assert sizes == sorted(sizes)
        sizes = [pg.pg_surrogate_scratch_floats(m, 20000) for m in range(1, 3000, 7)]
        assert sizes == sorted(sizes)


# ---------------------------------------------------------------- the binding

def test_the_binding_refuses_tensors_of_another_kind():
    d = pg.Logits(torch.zeros(3, 50))
    f = torch.zeros
    t = f(3, dtype=torch.int32)
    for bad in (dict(target=t.long()), dict(target=f(4, dtype=torch.int32)), dict(logp=f(3).double()), dict(logp=f(6)[::2]), dict(entropy=f(2)),
                dict(stats=f(3, 3)), dict(top_ids=f(3, 5)), dict(top_ids=f(3, 5, dtype=torch.int32), top_logp=f(3, 4)), dict(temperature=f(1))):
        args = {**dict(target=t, logp=f(3), scratch=f(100000)), **bad}
        with pytest.raises(AssertionError):
            pg.pg_token_logprobs(d, args.pop("target"), args.pop("logp"), args.pop("scratch"), **args)
    stats = f(3, 4)
    for out in (f(3, 50, dtype=torch.bfloat16), f(3, 49), f(2, 50), f(50, 3).t()):
        with pytest.raises(AssertionError):
            pg.pg_token_logprobs_backward(d, t, stats, out, g_logp=f(3))
        with pytest.raises(AssertionError):
            pg.pg_distill_backward(d, f(3, 2, dtype=torch.int32), f(3, 2), f(3, 8), f(3), out)
    for bad in (dict(ids=f(3, 2)), dict(values=f(3, 3)), dict(loss=f(4)), dict(stats=f(3, 4))):
        args = {**dict(ids=f(3, 2, dtype=torch.int32), values=f(3, 2), loss=f(3), scratch=f(100000)), **bad}
        with pytest.raises(AssertionError):
            pg.pg_distill_loss(d, args.pop("ids"), args.pop("values"), args.pop("loss"), args.pop("scratch"), **args)
    cu = f(4, dtype=torch.int32)
    for bad in (dict(old=f(9)), dict(adv=f(4)), dict(cu=cu[:3]), dict(g=f(9)), dict(objective=f(3).half()), dict(logp_ref=f(3)), dict(clipped=f(3))):
        args = {**dict(old=f(10), adv=f(3), cu=cu, objective=f(3), g=f(10)), **bad}
        with pytest.raises(AssertionError):
            pg.pg_token_surrogate(f(10), args.pop("old"), args.pop("adv"), args.pop("cu"), args.pop("objective"), args.pop("g"), 0.2, 0.2, 5, **args)


# ---------------------------------------------------------------- the oracle

def rows(seed, n=6, vocab=23):
    rng = np.random.default_rng(seed)
    return rng, rng.standard_normal((n, vocab)) * 2, rng.integers(0, vocab, size=n)


def test_oracles_log_probs_are_the_log_softmax():
    rng, z, target = rows(0)
    allow = rng.random(z.shape) < 0.7
    allow[np.arange(6), target] = True
    for r in range(6):
        got = ref.token_logprobs(z[r], target[r], 0.7, allow[r], 30)
        ln = torch.log_softmax(torch.from_numpy(z[r]) / 0.7 + torch.where(torch.from_numpy(allow[r]), 0.0, -math.inf), 0)
        assert abs(got["logp"] - float(ln[target[r]])) < 1e-13
        assert abs(got["entropy"] + float(torch.nansum(ln.exp() * ln))) < 1e-13
        order = [i for i in torch.argsort(-ln).tolist() if allow[r, i]]
        assert got["top_ids"].tolist() == order + [-1] * (30 - len(order))
    assert ref.token_logprobs(np.zeros(4), 2, n_top=3)["top_ids"].tolist() == [0, 1, 2]
    assert math.isnan(ref.token_logprobs(np.array([1.0, math.nan]), 0)["logp"])
    assert ref.token_logprobs(np.full(3, -math.inf), 0)["logp"] == -math.inf and ref.token_logprobs(np.zeros(3), -1)["logp"] == 0


def slope(f, z, way, h=1e-6):
    return (f(z + h * way) - f(z - h * way)) / (2 * h)


def test_oracles_gradients_are_the_slopes():
    rng, z, target = rows(1)
    allow = rng.random(z.shape) < 0.7
    allow[np.arange(6), target] = True
    for r in range(6):
        way = rng.standard_normal(z.shape[1])
        f = lambda x: 0.3 * ref.token_logprobs(x, target[r], 1.4, allow[r])["logp"] - 0.8 * ref.token_logprobs(x, target[r], 1.4, allow[r])["entropy"]  # noqa: E731
        d = ref.token_logprobs_gradient(z[r], target[r], 0.3, -0.8, 1.4, allow[r])
        assert abs(slope(f, z[r], way) - d @ way) < 1e-8
        ids = rng.permutation(23)[:7]
        ids[5], ids[6] = -1, ids[0]
        values = np.log(rng.dirichlet(np.ones(8))[:7])
        for tail in (False, True):
            for mask in (None, allow[r] | np.isin(np.arange(23), ids)):
                d = ref.distill(z[r], ids, values, tail, 1.4, mask)[1]
                assert abs(slope(lambda x: ref.distill(x, ids, values, tail, 1.4, mask)[0], z[r], way) - d @ way) < 1e-8


def test_oracles_distillation_is_the_divergence():
    rng, z, _ = rows(2)
    q = torch.log_softmax(torch.from_numpy(rng.standard_normal((6, 23))), 1)
    ids = np.arange(23)
    for r in range(6):
        want = float(torch.nn.functional.kl_div(torch.log_softmax(torch.from_numpy(z[r]), 0), q[r], log_target=True, reduction="sum"))
        for tail in (False, True):
            assert abs(ref.distill(z[r], ids, q[r].numpy(), tail)[0] - want) < 1e-12
        # a tail: the listed tokens and all others as one
        p = torch.softmax(torch.from_numpy(z[r]), 0)
        few = [3, 9, 1]
        a = torch.cat([q[r].exp()[few], (1 - q[r].exp()[few].sum())[None]])
        b = torch.cat([p[few], (1 - p[few].sum())[None]])
        assert abs(ref.distill(z[r], few, q[r].numpy()[few], True)[0] - float((a * (a / b).log()).sum())) < 1e-12


def test_oracles_objective_is_the_clipped_one():
    rng = np.random.default_rng(3)
    logp, old, x = (-rng.random(200) * 3 for _ in range(3))
    for adv in (1.3, -0.7, 0.0):
        t = torch.from_numpy(logp).requires_grad_()
        rho, log_ref = torch.exp(t - torch.from_numpy(old)), torch.from_numpy(x) - t
        kl = torch.exp(log_ref) - log_ref - 1
        want = (torch.minimum(rho * adv, rho.clamp(0.8, 1.3) * adv) - 0.1 * kl).mean()
        want.backward()
        got = ref.surrogate(logp, old, adv, 0.2, 0.3, x, 0.1)
        assert abs(got["objective"] - float(want.detach())) < 1e-13 and abs(got["kl"] - float(kl.detach().mean())) < 1e-13
        np.testing.assert_allclose(got["g_logp"], t.grad.numpy(), atol=1e-14)
        assert got["clipped"] == int(((rho > 1.3) if adv > 0 else (rho < 0.8) if adv < 0 else rho < 0).sum())
