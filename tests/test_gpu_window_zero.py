"""GPU tests of window attention with a window of 0: only the sinks are visible, and
only table entries of pages that hold a sink may be looked up."""

from __future__ import annotations

import numpy as np
import pytest

import window_model
from gpu_util import announce, require_gpu
from test_gpu_window import Case, both, ints

pytestmark = pytest.mark.gpu


class Seen(Case):
    """A case whose table has an entry only where the definition sees a token of the page."""

    def needed(self, n, m, t):
        return any(t in window_model.visible(p, self.window, self.sinks) for p in range(max(n - m, t), n))


# lens, news, hkv, group, dim, page, sinks
SHAPES = [
    ([60], [4], 2, 4, 64, 16, 5), ([200], [60], 2, 4, 64, 16, 5), ([100], [100], 1, 4, 128, 16, 5), ([77, 31], [3, 5], 1, 3, 128, 16, 17), ([64], [16], 1, 1, 64, 16, 20),
    ([96, 97, 95], [1, 1, 1], 2, 8, 64, 16, 5), ([130, 40], [1, 40], 2, 4, 128, 16, 33), ([60, 70], [4, 50], 1, 2, 64, 4, 6), ([90], [5], 1, 2, 128, 2, 3), ([90], [70], 1, 2, 64, 1, 3),
    ([257], [129], 1, 2, 128, 64, 70), ([65], [9], 1, 1, 64, 8, 64), ([90], [80], 1, 4, 64, 16, 1000), ([90], [4], 1, 4, 64, 16, 1000), ([33], [17], 2, 1, 64, 16, 0),
    ([2500, 48], [2, 48], 1, 4, 64, 16, 2000), ([1500, 900], [700, 1], 2, 4, 128, 32, 100),
]


@pytest.mark.parametrize("dtype,lens,news,hkv,group,dim,page,sinks", both(*SHAPES))
def test_only_the_sinks_are_seen(dtype, lens, news, hkv, group, dim, page, sinks):
    require_gpu()
    announce(f"window 0 {dtype} lens={lens} news={news} hkv={hkv} g={group} d={dim} page={page} s={sinks}")
    c = Seen(sum(lens) + sinks, dtype, lens, news, hkv, group, dim, page, 0, sinks)
    for n, row in zip(lens, c.table):
        held = {t // page for t in range(min(sinks, n))}
        assert all((int(p) >= 0) == (e in held) for e, p in enumerate(row))
    c.check(c.run())


@pytest.mark.parametrize("n", [32, 33, 47, 48, 64, 100])
def test_one_new_token_beside_many_rows(n):
    """The only sequence of a buffer for more than 16 rows: one new token, at any place of its group of 16."""
    import torch

    from paper_2412_15803_amd import wq

    require_gpu()
    c = Seen(n, "float16", [n], [1], 2, 4, 64, 16, 0, 5)
    q = torch.cat([c.q, torch.zeros((7, 8, 64), dtype=c.kind, device="cuda")])
    out = torch.full_like(q, 7.0)
    wq.window_attention(q, c.k, c.v, ints(c.table), ints(c.lens), out, c.scale, n, 0, sinks=5, q_starts=ints([0, 1]), max_query_len=8)
    c.check(out[:1])
    assert bool((out[1:] == 7.0).all())


@pytest.mark.parametrize("news", [1, 3, 40])
def test_after_the_pages_behind_the_sinks_are_given_back(news):
    """cache_free with the same window and sinks leaves what the attention needs."""
    from paper_2412_15803_amd import wq

    require_gpu()
    c = Case(8, "bfloat16", [150], [news], 1, 8, 64, 16, 200, 0)
    c.window, c.sinks = 0, 5
    table, refs = ints(c.table), ints(np.ones(c.k.shape[0]))
    wq.cache_free(table, refs, ints(c.lens), ints([0]), 16, window=0, sinks=5)
    c.table = table.cpu().numpy().astype(np.int64)
    assert (c.table[0] >= 0).tolist() == [True] + [False] * 9
    c.check(c.run())
