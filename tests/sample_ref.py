"""Sampling in 64 bits on the CPU, written from its definition, for the tests."""
import math

import numpy as np


def kept(x, T, k, p, q):
    """(ids in the order of what is kept, their weights): x a row's logits in 64 bits."""
    x = np.where(np.isnan(x), -np.inf, x)
    if not (x > -np.inf).any():
        return np.zeros(0, int), np.zeros(0)
    order = np.lexsort((np.arange(len(x)), -x))
    top = x[order[0]]
    if not T > 0:
        return order[:1], np.ones(1)
    order = order[x[order] > -np.inf]
    if top == np.inf:
        w = (x[order] == np.inf).astype(float)
    else:
        w = np.exp((x[order] - top) / T)
    if 0 < k < len(x):
        order, w = order[:k], w[:k]
    if p < 1:
        before = np.concatenate([[0.0], np.cumsum(w)[:-1]])
        n = max(1, int((before < p * math.fsum(w)).sum()))
        order, w = order[:n], w[:n]
    on = w >= min(q, 1.0) if q > 0 else np.ones(len(w), bool)
    return order[on], w[on]


def sample(x, u, T=1.0, k=0, p=1.0, q=0.0):
    """(token, its log-probability)"""
    ids, w = kept(x, T, k, p, q)
    if not len(ids):
        return -1, -math.inf
    u = 0.0 if not u > 0 else min(u, 1 - 2.0 ** -30)
    at = np.argsort(ids)
    ids, w = ids[at], w[at]
    run = np.cumsum(w)
    i = int(np.argmax((run > u * run[-1]) & (w > 0)))
    return int(ids[i]), math.log(w[i] / math.fsum(w))
