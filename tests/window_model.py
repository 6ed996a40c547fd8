"""Window attention row by row in 64 bits, straight from the definition, on NumPy
arrays: what the device operator is compared with."""

from __future__ import annotations

import numpy as np


def visible(place, window, sinks):
    t = np.arange(place + 1)
    return t[(t < sinks) | (t > place - window)]


def attend(q, k_cache, v_cache, table, lens, starts, scale, window, sinks):
    """(outputs, sum of w |V|, largest scale * sum |q K|); q [T, HQ, D] and the
    caches [pages, HKV, P, D] float64."""
    page, hkv = k_cache.shape[2], k_cache.shape[1]
    total, hq, dim = q.shape
    group = hq // hkv
    out, size = np.zeros(q.shape), np.zeros(q.shape)
    most = 0.0
    for s, n in enumerate(lens):
        first, end = (s, s + 1) if starts is None else (starts[s], starts[s + 1])
        for row in range(first, end):
            t = visible(n - (end - row), window, sinks)
            if len(t) == 0:
                continue
            pages = np.asarray(table[s])[t // page]
            for h in range(hkv):
                k, v = k_cache[pages, h, t % page], v_cache[pages, h, t % page]
                qs = q[row, h * group:(h + 1) * group]
                a = scale * (qs @ k.T)
                most = max(most, abs(scale) * float(np.max(np.abs(qs) @ np.abs(k).T)))
                w = np.exp(a - a.max(-1, keepdims=True))
                w /= w.sum(-1, keepdims=True)
                out[row, h * group:(h + 1) * group] = w @ v
                size[row, h * group:(h + 1) * group] = w @ np.abs(v)
    return out, size, most
