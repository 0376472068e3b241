"""Sampling behind top-k, top-p and min-p on the host, from its definition: weights in float64, sums in whole numbers (64 bits hold those of 2^31 tokens)."""
import math

import numpy as np


def weights(l, tau):
    """(l / tau - max / tau, floor(exp of it * 2^32)) of a row with something above -infinity and no NaN."""
    top = l.max()
    with np.errstate(all="ignore"):
        z = np.where(l == top, 0.0, l / tau - top / tau)
        w = np.floor(np.exp(z) * 2.0 ** 32)
    return z, np.where((l == -math.inf) | ~(z >= -1e300), 0.0, w).astype(np.int64)


def choose(l, tau=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """l: float64 values of a row -> (kept indices, most likely first; z; W), or (None, ..) for a row with a NaN."""
    l = np.asarray(l, np.float64)
    tau, top_p, min_p = float(np.float32(tau)), float(np.float32(top_p)), float(np.float32(min_p))
    if np.isnan(l).any():
        return None, None, None
    if l.max() == -math.inf:
        return np.zeros(0, np.int64), None, None
    greedy = not tau > 0
    z, W = weights(l, 1.0 if greedy else tau)
    order = np.argsort(-l, kind="stable")
    order = order[l[order] > -math.inf]
    if greedy:
        return order[:1], z, W
    if top_k > 0:
        order = order[:top_k]
    if top_p < 1:
        share, run = int(math.floor(max(top_p, 0.0) * 2 ** 31)), np.cumsum(W[order])
        aim = max(-(-share * int(run[-1]) // 2 ** 31), 1)
        order = order[run - W[order] < aim]
    if min_p > 0:
        order = order[W[order] >= int(math.floor(min(min_p, 1.0) * 2 ** 32))]
    return order, z, W


def draw(l, u, **ask):
    """(token, (log-probability among the kept, in the whole row), number of kept tokens)"""
    kept, z, W = choose(l, **ask)
    if kept is None:
        return -1, (math.nan, math.nan), 0
    if not len(kept):
        return -1, (-math.inf, -math.inf), 0
    by_index = np.sort(kept)
    run = np.cumsum(W[by_index])
    S = int(run[-1])
    j = int(by_index[np.searchsorted(run, (int(u) * S) >> 32, side="right")])
    return j, (z[j] - math.log(S / 2 ** 32), z[j] - math.log(int(W.sum()) / 2 ** 32)), len(kept)
