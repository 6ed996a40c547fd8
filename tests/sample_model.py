"""The choice of a word by chance in float64, word by word in its order: what the
device operator is compared with."""

from __future__ import annotations

import math

import numpy as np


def stays(x, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """Weight of each word of x (float64) that stays, 0 for the others; None where
    no word takes part.  A temperature of 0 leaves the best word."""
    part = [i for i in range(len(x)) if not math.isnan(x[i]) and x[i] != -math.inf]
    if not part:
        return None
    order = sorted(part, key=lambda i: (-x[i], i))
    top = x[order[0]]
    out = np.zeros(len(x))
    if not temperature > 0:
        out[order[0]] = 1.0
        return out
    if math.isinf(top):
        w = {i: 1.0 if x[i] == top else 0.0 for i in order}
    else:
        w = {i: math.exp((x[i] - top) / temperature) for i in order}
    if top_k > 0:
        order = order[:top_k]
    if top_p < 1:
        total, sum_, kept = math.fsum(w[i] for i in order), 0.0, []
        for i in order:
            kept.append(i)
            sum_ += w[i]
            if sum_ >= top_p * total:
                break
        order = kept
    if min_p > 0:
        order = [i for i in order if w[i] >= min(min_p, 1.0)]
    for i in order:
        out[i] = w[i]
    return out


def choose(weights, u):
    """The word at which the weights' sum passes u of the total, and its share."""
    if weights is None:
        return -1, 0.0
    sums = np.cumsum(weights)
    i = min(int(np.searchsorted(sums, u * sums[-1], side="right")), int(np.flatnonzero(weights)[-1]))
    return i, weights[i] / sums[-1]


def clear_of_borders(weights, u, margin=1e-9):
    """Whether u lies further than `margin` of the total from every border between words."""
    sums = np.cumsum(weights) / np.sum(weights)
    return bool(np.abs(sums[weights > 0][:-1] - u).min(initial=1.0) > margin)
