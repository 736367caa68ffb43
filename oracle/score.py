"""Scores of given tokens and the embedding's gradient from their definitions, in
64 bits (numpy); share nothing with the HIP path."""
from __future__ import annotations

import math
from typing import NamedTuple

import numpy as np

INF = math.inf


class Scored(NamedTuple):
    logp: float
    entropy: float
    words: np.ndarray    # the k first in (x descending, word ascending)
    word_logp: np.ndarray
    log_p: np.ndarray    # of every word


def score(x, token: int, k: int = 0, temperature: float = 1.0) -> Scored:
    """One row. token < 0: none."""
    x = np.asarray(x, dtype=np.float64)
    if token < 0:
        return Scored(0.0, 0.0, np.full(k, -1), np.zeros(k), np.zeros(x.size))
    top = x.max()
    if not math.isfinite(top):  # NaN, +inf, or no word at all
        nan = np.full(x.size, math.nan)
        return Scored(math.nan, math.nan, np.full(k, -1), nan[:k], nan)
    s = (x - top) / temperature  # from the largest: a row of far logits loses nothing
    log_p = s - math.log(np.exp(s).sum())
    p = np.exp(log_p)
    entropy = -float(np.sum(p[p > 0] * log_p[p > 0]))
    words = np.lexsort((np.arange(x.size), -(x + 0.0)))[:k]
    return Scored(float(log_p[token]), entropy, words, log_p[words], log_p)


def score_gradient(x, token: int, dlogp: float, dentropy: float, temperature: float = 1.0):
    """The gradient of dlogp * logp + dentropy * entropy, through the softmax's Jacobian:
    dp_j/dx_i = p_j (1{i = j} - p_i) / temperature."""
    x = np.asarray(x, dtype=np.float64)
    if token < 0 or (dlogp == 0 and dentropy == 0):
        return np.zeros(x.size)
    r = score(x, token, 0, temperature)
    p = np.exp(r.log_p)
    with np.errstate(all="ignore"):
        # entropy's derivative by p_j is -(log p_j + 1), whose 1 the Jacobian takes out
        v = np.where(p > 0, -p * r.log_p, 0.0) * dentropy
    g = v - p * v.sum() - dlogp * p
    g[token] += dlogp
    return g / temperature


def embed_sums(tokens, dout, vocab: int, scale: float = 1.0):
    """(G, A, counts): the table's gradient, the sum of magnitudes behind each of its
    elements, and each word's tokens. One token after the other."""
    dout = np.asarray(dout, dtype=np.float64)
    g = np.zeros((vocab, dout.shape[1]))
    a = np.zeros_like(g)
    counts = np.zeros(vocab, np.int64)
    for i, t in enumerate(np.asarray(tokens).ravel().tolist()):
        if 0 <= t < vocab:
            g[t] += dout[i]
            a[t] += np.abs(dout[i])
            counts[t] += 1
    return g * scale, a * abs(scale), counts
