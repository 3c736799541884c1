"""Plain fp64 oracle of what a token policy learns from (test infrastructure only): log-probs with entropy and alternatives,
divergence from a teacher's list, the clipped objective, and their gradients.  Written from the definitions in the C header, one row and
one sequence at a time, on values in fp64 (what lies there in fp32 or bf16, without rounding)."""
import numpy as np


def softmax(z, temperature=1.0, allow=None):
    """(y, ln p, ln of the softmax's denominator, bad): y = z / T with -inf where a token is not allowed."""
    z = np.asarray(z, dtype=np.float64)
    t = 1.0 if temperature == 0 else float(temperature)
    open_ = np.ones(z.shape, dtype=bool) if allow is None else np.asarray(allow, dtype=bool)
    bad = not (0 <= temperature < np.inf) or bool(np.any(np.isnan(z[open_]) | (z[open_] == np.inf)))
    y = np.where(open_, z, -np.inf) / (1.0 if bad else t)
    if bad:
        return y, np.full(z.shape, np.nan), np.nan, True
    top = y.max()
    if top == -np.inf:
        return y, np.full(z.shape, -np.inf), -np.inf, False
    ln_sum = np.log(np.exp(y - top).sum())
    return y, (y - top) - ln_sum, top + ln_sum, False            # ln p in two steps: far from 0 the denominator takes no ln_sum


def token_logprobs(z, target, temperature=1.0, allow=None, n_top=0):
    """dict(logp, entropy, lse, top_ids, top_logp) of one row; target None: there is none."""
    ids, values = np.full(n_top, -1), np.full(n_top, -np.inf)
    if target == -1:
        return dict(logp=0.0, entropy=0.0, lse=None, top_ids=ids, top_logp=values)
    y, ln, lse, bad = softmax(z, temperature, allow)
    if bad:
        return dict(logp=np.nan, entropy=np.nan, lse=np.nan, top_ids=ids, top_logp=np.full(n_top, np.nan))
    p = np.exp(ln)
    entropy = -np.sum(p[p > 0] * ln[p > 0])
    order = np.lexsort((np.arange(len(y)), -np.where(np.isfinite(y), np.asarray(z, dtype=np.float64), -np.inf)))[:n_top]
    order = order[np.isfinite(y[order])]
    ids[:len(order)], values[:len(order)] = order, ln[order]
    logp = None if target is None else ln[target] if 0 <= target < len(y) else np.nan
    return dict(logp=logp, entropy=entropy, lse=lse, top_ids=ids, top_logp=values)


def token_logprobs_gradient(z, target, g_logp, g_entropy, temperature=1.0, allow=None):
    if target == -1 or (g_logp == 0 and g_entropy == 0):
        return np.zeros(len(z))
    y, ln, lse, bad = softmax(z, temperature, allow)
    there = y > -np.inf if not bad else (np.ones(len(z), dtype=bool) if allow is None else np.asarray(allow, dtype=bool)) & (np.asarray(z) != -np.inf)
    if bad or (target is not None and not 0 <= target < len(z)):
        return np.where(there, np.nan, 0.0)
    p = np.exp(ln)
    h = -np.sum(p[p > 0] * ln[p > 0])
    d = np.zeros(len(z))
    d[there] = -g_logp * p[there] - g_entropy * p[there] * (ln[there] + h)
    if target is not None and there[target]:
        d[target] += g_logp
    return d / (1.0 if temperature == 0 else temperature)


def distill(z, ids, values, tail, temperature=1.0, allow=None):
    """(loss, gradient with respect to z) of one row."""
    vocab = len(z)
    seen, q = [], []
    for i, v in zip(ids, values):
        if 0 <= i < vocab and i not in seen:
            seen.append(int(i))
            q.append(float(v))
    y, ln, lse, bad = softmax(z, temperature, allow)
    nothing = 0.0, np.zeros(vocab)
    if not seen or (not bad and lse == -np.inf):
        return nothing
    q = np.array(q)
    there = (np.ones(vocab, dtype=bool) if allow is None else np.asarray(allow, dtype=bool)) & (np.asarray(z) != -np.inf)
    wrong = bool(np.any(np.isnan(q) | (q == np.inf)))
    if not tail and not wrong and q.max() == -np.inf:
        return nothing
    if bad or wrong:
        return np.nan, np.where(there, np.nan, 0.0)
    rest = np.ones(vocab, dtype=bool)
    rest[seen] = False
    p = np.exp(ln)
    p_rest = np.sum(p[rest])
    if tail:
        w = np.exp(q)
        q_rest = max(0.0, 1.0 - np.sum(w)) if np.any(there & rest) else 0.0
    else:
        w = np.exp(q - q.max())
        w, q_rest = w / w.sum(), 0.0
    with np.errstate(divide="ignore", invalid="ignore"):
        loss = sum(a * (np.log(a) - ln[i]) for a, i in zip(w, seen) if a > 0)
        if q_rest > 0:
            loss += q_rest * (np.log(q_rest) - np.log(p_rest))
    everything = np.sum(w) + q_rest
    d = everything * p
    if q_rest > 0:
        d[rest] -= q_rest / p_rest * p[rest]
    d[seen] -= w
    d = np.where(there, d, 0.0)
    return loss, d / (1.0 if temperature == 0 else temperature)


def surrogate(logp, old, adv, clip_low, clip_high, ref=None, kl_coef=0.0, weight=None):
    """dict(objective, kl, clipped, g_logp) of one sequence."""
    logp, old = np.asarray(logp, dtype=np.float64), np.asarray(old, dtype=np.float64)
    n = len(logp)
    if n == 0:
        return dict(objective=0.0, kl=0.0, clipped=0, g_logp=np.zeros(0))
    w = 1.0 / n if weight is None else float(weight)
    with np.errstate(over="ignore", invalid="ignore"):
        rho = np.exp(logp - old)
        a = float(adv)
        cut = (rho > 1 + clip_high) & (a > 0) | (rho < 1 - clip_low) & (a < 0)
        ra = np.zeros(n) if a == 0 else rho * a
        term = np.where(cut, a * (1 + clip_high if a > 0 else 1 - clip_low), ra)
        g = np.where(cut, 0.0, ra)
        kl = np.zeros(n)
        if ref is not None:
            x = np.asarray(ref, dtype=np.float64) - logp
            kl = np.where(np.expm1(x) == np.inf, np.inf, np.expm1(x) - x)
            if kl_coef != 0:                               # 0 e^1000 is 0, which fp64 would make no number
                term, g = term - kl_coef * kl, g + kl_coef * np.expm1(x)
    return dict(objective=w * term.sum(), kl=kl.mean(), clipped=int(cut.sum()), g_logp=w * g)
