"""Row operators from their definitions, in 64 bits (numpy): top logits,
distillation on (idx, val) lists, verification of drafted tokens. One row or
one sequence at a time; shares nothing with the HIP path."""
from __future__ import annotations

import math
from typing import NamedTuple, Optional

import numpy as np

INF = math.inf


def logsumexp(x) -> float:
    x = np.asarray(x, dtype=np.float64)
    if x.size == 0:
        return -INF
    m = x.max()
    if not math.isfinite(m):
        return float(m)  # -inf: nothing; +inf and NaN stay
    return float(m + np.log(np.sum(np.exp(x - m))))


def top(x, k: int, temperature: float = 1.0):
    """(idx, val, tail): the k words first in (x descending, word ascending),
    in ascending order, and the log-mass of the others."""
    x = np.asarray(x, dtype=np.float64) + 0.0  # -0 -> +0 for the comparison only
    order = np.lexsort((np.arange(x.size), -x))
    idx = np.sort(order[:k])
    rest = np.delete(x, idx)
    return idx.astype(np.int32), x[idx], logsumexp(rest / temperature)


class Distilled(NamedTuple):
    loss: float
    grad: np.ndarray
    p: np.ndarray       # teacher's probabilities of the listed words
    p_rest: float
    q: np.ndarray       # student's probabilities
    q_rest: float


def distill(z, idx, val, tail: float = -INF, weight: float = 1.0,
            temperature: float = 1.0) -> Distilled:
    """One row; idx and val hold the used entries."""
    z = np.asarray(z, dtype=np.float64)
    idx = np.asarray(idx, dtype=np.int64)
    t = np.asarray(val, dtype=np.float64) / temperature
    if weight == 0.0 or idx.size == 0:
        return Distilled(0.0, np.zeros(z.size), np.zeros(idx.size), 0.0, np.zeros(z.size), 0.0)
    # from the row's largest logit: a row of nothing but a mask's value (-3e38,
    # say) would lose the logarithm of its sum even in 64 bits
    top = z.max()
    s = (z - top) / temperature if math.isfinite(top) else z / temperature
    lt = logsumexp(np.append(t, tail))
    lz = logsumexp(s)
    if not math.isfinite(lt) or not math.isfinite(lz):
        nan = np.full(z.size, math.nan)
        return Distilled(math.nan, nan, nan[: idx.size], math.nan, nan, math.nan)
    lp, lq = t - lt, s - lz
    lpr = tail - lt
    outside = np.ones(z.size, bool)
    outside[idx] = False
    lqr = logsumexp(lq[outside])
    loss = 0.0
    for a, b in zip(lp, lq[idx]):
        if a > -INF:
            loss += math.exp(a) * (a - b)
    if lpr > -INF:
        loss += math.exp(lpr) * (lpr - lqr)
    p, q = np.exp(lp), np.exp(lq)
    grad = q.copy()
    grad[idx] -= p
    if lpr > -INF and lqr > -INF:
        # q (1 - p_r / q_r) = q - p_r (q / q_r), the last a softmax of its own
        grad[outside] -= math.exp(lpr) * softmax(z[outside] / temperature)
    return Distilled(loss * weight * temperature ** 2, grad * weight * temperature, p,
                     math.exp(lpr), q, math.exp(lqr))


class Verified(NamedTuple):
    accepted: int
    tokens: list
    logp: list
    margin: float       # smallest relative distance of a decision from the other outcome


def softmax(x):
    x = np.asarray(x, dtype=np.float64)
    m = x.max()
    if m == -INF:
        return np.zeros(x.size)
    e = np.exp(x - m)
    return e / e.sum()


def verify(target, drafts, tokens, uniform, noise, length: Optional[int] = None,
           temperature: float = 1.0) -> Verified:
    """One sequence: target (draft + 1, V), drafts (draft, V)."""
    draft = len(tokens)
    m = draft if length is None else length
    out, logp, margin, n = [], [], INF, 0
    while n < m:
        p, q = softmax(target[n] / temperature), softmax(drafts[n] / temperature)
        x = int(tokens[n])
        if not 0 <= x < p.size:
            break
        a, b = float(uniform[n]) * q[x], p[x]
        if a != b and not (math.isnan(a) or math.isnan(b)):
            margin = min(margin, abs(a - b) / max(a, b))
        if not a < b:
            break
        out.append(x)
        logp.append(math.log(p[x]))
        n += 1
    p = softmax(target[n] / temperature)
    r = p
    if n < m:
        r = np.maximum(p - softmax(drafts[n] / temperature), 0.0)
        if not np.any(r > 0):
            r = p
    with np.errstate(all="ignore"):
        score = np.where(r > 0, r / np.asarray(noise, dtype=np.float64), -1.0)
    y = int(np.argmax(score)) if np.any(score > 0) else -1
    if y >= 0:
        others = np.delete(score, y)
        if others.size and others.max() > 0 and others.max() != score[y]:
            # the quotient's own rounding grows where p - q cancels
            part = r[y] / p[y] if n < m else 1.0
            margin = min(margin, (score[y] - others.max()) / score[y] * part)
    out.append(y)
    logp.append(math.log(p[y]) if y >= 0 else 0.0)
    pad = draft - n
    return Verified(n, out + [-1] * pad, logp + [0.0] * pad, margin)
