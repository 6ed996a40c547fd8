"""The step from logits to a token in 64 bits, word by word: what the device
operator is compared with."""

from __future__ import annotations

import math


def process(x, mask=None, history=(), prompt=0, repetition=1.0, frequency=0.0, presence=0.0, bias=()):
    """(values, best word) of one row: x a list of floats, mask a list of truth
    values, bias a list of (word, value)."""
    out, counts, seen = [], {}, set()
    for i, w in enumerate(history):
        seen.add(w)
        if i >= prompt:
            counts[w] = counts.get(w, 0) + 1
    listed = dict(bias)  # the later entry of a word holds
    best = -1
    for w, v in enumerate(x):
        if w in seen:
            v = v / repetition if v > 0 else v * repetition
            v = v - frequency * counts.get(w, 0)
            if counts.get(w, 0):
                v = v - presence
        if w in listed:
            v = v + listed[w]
        if mask is not None and not mask[w]:
            out.append(-math.inf)
            continue
        out.append(v)
        if not math.isnan(v) and (best < 0 or v > out[best]):
            best = w
    return out, best
