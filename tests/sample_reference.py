"""Sampling by its definition, row by row on the host in 64 bits."""
from __future__ import annotations

import math

import numpy as np


def kept_tokens(logits, temperature, top_k=0, top_p=1.0, min_p=0.0):
    """The tokens that may be drawn, in the order of falling logits, and the weights of all tokens."""
    logits = np.where(np.isnan(logits), -np.inf, logits)
    order = np.lexsort((np.arange(logits.size), -logits))
    top = logits[order[0]]
    if top == -np.inf:
        return order[:0], np.zeros(logits.size)
    warm = temperature > 0
    with np.errstate(invalid="ignore", over="ignore"):
        w = np.where(logits == top, 1.0, np.exp((logits - top) / (temperature if warm and np.isfinite(top) else 1.0)))
    m = int(np.count_nonzero(logits > -np.inf))
    if not warm:
        m = 1
    if top_k > 0:
        m = min(m, int(top_k))
    if min_p > 0:
        m = min(m, int(np.count_nonzero(w[order] >= min_p)))
    m = max(m, 1)
    if top_p < 1:
        upto = np.cumsum(w[order[:m]])
        m = min(m, int(np.searchsorted(upto, top_p * upto[-1], side="left")) + 1)
    return order[:m], w


def token_of(logits, u, *settings):
    """The token of a row and the log of its probability."""
    order, w = kept_tokens(logits, *settings)
    if not len(order):
        return -1, -math.inf
    kept = np.sort(order)
    kept = kept[w[kept] > 0]
    upto = np.cumsum(w[kept])
    u = u if u > 0 else 0.0
    token = kept[min(int(np.searchsorted(upto, u * upto[-1], side="right")), len(kept) - 1)]
    return int(token), math.log(w[token]) - math.log(math.fsum(w[kept]))
