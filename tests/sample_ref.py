"""Sampling with temperature, top-k, top-p and min-p from a given uniform, in 64 bits, from the definition."""
import math

import numpy as np


def weights(x, tau, top_k=0, top_p=1.0, min_p=0.0):
    """What stays of a row, as weights by id (0: does not stay); None for a row without a token."""
    x = np.asarray(x, np.float32)
    x = np.where(np.isnan(x), -np.inf, np.where(x == np.inf, np.finfo(np.float32).max, x)).astype(np.float64)
    order = np.lexsort((np.arange(x.size), -x))          # falling logits, equal ones by id
    M = x[order[0]]
    if M == -np.inf:
        return None
    w = np.zeros(x.size)
    if tau == 0:
        w[order[0]] = 1.0
        return w
    d = (M - x) / float(tau)
    w = np.where((d <= 40 * math.log(2)) & (x > -np.inf), np.exp(-d), 0.0)
    s = w[order]
    rank = np.arange(x.size)
    if top_k > 0:
        s = np.where(rank < top_k, s, 0.0)
    front = np.concatenate([[0.0], np.cumsum(s)[:-1]])
    stays = s >= min_p
    if top_p < 1:
        stays &= front < float(top_p) * s.sum()
    out = np.zeros(x.size)
    out[order] = np.where(stays, s, 0.0)
    return out


def token(x, u, tau, top_k=0, top_p=1.0, min_p=0.0):
    w = weights(x, np.float32(tau), int(top_k), np.float32(top_p), np.float32(min_p))
    if w is None:
        return -1
    u = np.float32(u)
    u = 0.0 if not u > 0 else min(float(u), 1.0 - 2.0 ** -24)
    c = np.cumsum(w)
    at = int(np.searchsorted(c, u * c[-1], side="right"))
    return min(at, int(np.nonzero(w)[0][-1]))


def tokens(x, u, tau, top_k=0, top_p=1.0, min_p=0.0):
    """x [batch, T, V], u [batch, T], options [batch] or numbers."""
    batch, T, _ = x.shape
    o = [np.broadcast_to(np.asarray(v), (batch,)) for v in (tau, top_k, top_p, min_p)]
    return np.array([[token(x[b, i], u[b, i], *(v[b] for v in o)) for i in range(T)] for b in range(batch)], np.int32)
