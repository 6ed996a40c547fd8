"""GPU tests of small softmax weights in window attention: one token outweighs all
others by many nats but has zero values, so that the output is what the others add.

Bounds.  A fp16 value is off by at most 2^-25 below 2^-14, and weights are formed so
that the largest is at least 2^7 (include/wq_window.h).  So to the bound that the other
tests derive come 2^-25 / 2^7 = 2^-32 of every visible |V| where a sequence's rows are
more than 16.  Up to 16 rows a weight's rounding error is multiplied too, 2^11 times as
fine: 2^-43.  bfloat16 has the range of fp32, and nothing is added."""

from __future__ import annotations

import numpy as np
import pytest

import window_model
from gpu_util import announce, require_gpu
from test_gpu_window import BOUND, Case

pytestmark = pytest.mark.gpu

DIM = 64


def dominated(dtype, n, news, group, page, window, sinks, gaps, at, seed=1, value=1.0):
    """Every key scores 0 but those of the tokens `at` (by rows' heads: gaps[h % len]), whose
    values are 0; the others' are `value` in half of the dims and random in the rest."""
    import torch

    c = Case(seed, dtype, [n], [news], 1, group, DIM, page, window, sinks, scale=1.0)
    c.k[:] = 0.0
    c.v *= value
    c.v[..., :DIM // 2] = value
    for t in at:
        p = int(c.table[0][t // page])
        c.k[p, :, t % page] = 1.0
        c.v[p, :, t % page] = 0.0
    for h in range(group):  # 64 equal products of gap / 64, exact in both types
        c.q[:, h] = gaps[h % len(gaps)] / DIM
    c.k64, c.v64, c.q64 = (torch.nan_to_num(x.double()).cpu().numpy() for x in (c.k, c.v, c.q))
    return c


def check(c):
    want, size, most = window_model.attend(c.q64, c.k64, c.v64, c.table, c.lens, c.starts, c.scale, c.window, c.sinks)
    assert most <= 60.0
    got = c.run().double().cpu().numpy()
    n, news, group = c.lens[0], c.news[0], c.q.shape[1]
    each = 0.0 if c.dtype == "bfloat16" else 2.0 ** -43 if news * group <= 16 else 2.0 ** -32
    bound = BOUND[c.dtype] * size + 1e-6
    for row in range(news):
        t = window_model.visible(n - news + row, c.window, c.sinks)
        v = c.v64[np.asarray(c.table[0])[t // c.page], 0, t % c.page]
        bound[row] += each * np.abs(v).sum(0)
    assert np.isfinite(got).all()
    off = np.abs(got - want) / bound
    print("largest share of the bound", float(off.max()))
    assert off.max() <= 1.0, (float(off.max()), np.unravel_index(off.argmax(), off.shape))


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("news,group", [(1, 4), (4, 4), (16, 1), (5, 4), (130, 2)])
@pytest.mark.parametrize("n", [1024, 8192])
@pytest.mark.parametrize("gap", [10.0, 14.0, 17.5, 20.0])
def test_a_first_token_that_outweighs_the_rest(dtype, news, group, n, gap):
    require_gpu()
    announce(f"weights {dtype} n={n} news={news} g={group} gap={gap}")
    check(dominated(dtype, n, news, group, 16, 1 << 20, 4, [gap], [0]))


@pytest.mark.parametrize("news,group,page", [(1, 2, 16), (3, 4, 4), (60, 4, 16), (60, 4, 4)])
@pytest.mark.parametrize("at", [0, 700, 1990])
def test_rows_of_different_gaps(news, group, page, at):
    """The token first, in the middle and late, in heads that it outweighs by more or less, or in which it is least."""
    require_gpu()
    announce(f"weights at={at} news={news} g={group} page={page}")
    check(dominated("float16", 2100, news, group, page, 2050, 70, [17.5, -3.0, 12.0, 0.0], [at]))


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("news,group,page", [(1, 4, 16), (4, 4, 16), (16, 1, 4), (130, 2, 16)])
@pytest.mark.parametrize("n", [960, 1024, 8192])
@pytest.mark.parametrize("gap", [10.0, 14.0, 17.5, 20.0])
def test_tokens_that_outweigh_the_rest_wherever_the_work_is_cut(dtype, news, group, page, n, gap):
    """One in every 32 tokens, so that whoever takes a part of the sequence meets one; the others' values are large."""
    require_gpu()
    announce(f"weights {dtype} n={n} news={news} g={group} page={page} gap={gap} every 32")
    check(dominated(dtype, n, news, group, page, 1 << 20, 4, [gap], range(0, n, 32), value=1000.0))


@pytest.mark.parametrize("news", [1, 40])
def test_weights_up_to_the_largest(news):
    """Scores that rise along the sequence by less than moves the reference: weights reach the top of the range."""
    import torch

    require_gpu()
    n = 640
    c = dominated("float16", n, news, 4, 16, 1 << 20, 0, [5.5], [0])
    rise = torch.linspace(0, 1, n).half()  # scores 0 .. 5.5 nats, just below 2^8
    for t in range(n):
        p = int(c.table[0][t // 16])
        c.k[p, :, t % 16] = rise[t].item()
        c.v[p, :, t % 16] = 1.0
    c.k64, c.v64 = (torch.nan_to_num(x.double()).cpu().numpy() for x in (c.k, c.v))
    check(c)
