"""GPU tests of window attention against the 64-bit model, within the bound that
its header states.

The bound, per element: e * sum_t w_t |V_t[d]| + 1e-6.  A weight's rounding to the
values' type is relative 2^-11 (bfloat16: 2^-8) and so is the output's (of at most
sum w |V|, 2^-11 and 2^-9 ... 2^-8); an fp32 score is off by at most 130 * 2^-24 *
60 = 4.7e-4 in the exponent, which moves a weight and its normalisation by as much
each.  2^-11 + 2^-11 + 2 * 4.7e-4 = 1.9e-3 < 3e-3 and 2^-8 + 2^-8 + 9.4e-4 =
8.8e-3 < 2e-2."""

from __future__ import annotations

import math

import numpy as np
import pytest

import window_model
from gpu_util import announce, require_gpu

pytestmark = pytest.mark.gpu

BOUND = {"float16": 3e-3, "bfloat16": 2e-2}


def ints(a):
    import torch

    return torch.from_numpy(np.ascontiguousarray(np.asarray(a, dtype=np.int32))).cuda()


class Case:
    """Sequences of `lens` tokens, the last `news` of them new, in a cache whose
    unused slots and pages hold NaN and whose unseen pages have no table entry."""

    def __init__(self, seed, dtype, lens, news, hkv, group, dim, page, window, sinks, scale=None, values="normal"):
        import torch

        g = torch.Generator().manual_seed(seed)
        rng = np.random.default_rng(seed)
        self.kind = getattr(torch, dtype)
        self.dtype, self.lens, self.news, self.window, self.sinks, self.page = dtype, list(lens), list(news), window, sinks, page
        self.scale = 1.0 / math.sqrt(dim) if scale is None else scale
        width = max(1, max(-(-n // page) for n in lens))
        used = [[e for e in range(-(-n // page)) if any(self.needed(n, m, t) for t in range(e * page, min(n, e * page + page)))] for n, m in zip(lens, news)]
        pages = max(1, sum(map(len, used))) + 2
        order = rng.permutation(pages)
        self.table = np.full((len(lens), width), -1, dtype=np.int64)
        k = torch.full((pages, hkv, page, dim), math.nan, dtype=torch.float64)
        v = torch.full((pages, hkv, page, dim), math.nan, dtype=torch.float64)
        at = 0
        for s, entries in enumerate(used):
            for e in entries:
                p = int(order[at])
                at += 1
                self.table[s, e] = p
                for t in range(e * page, min(lens[s], e * page + page)):
                    if self.needed(lens[s], news[s], t):
                        k[p, :, t % page] = torch.randn((hkv, dim), generator=g, dtype=torch.float64)
                        v[p, :, t % page] = torch.randn((hkv, dim), generator=g, dtype=torch.float64)
        if values == "integers":
            v = torch.round(v * 4)
        self.starts = np.concatenate([[0], np.cumsum(news)]) if any(n != 1 for n in news) else None
        total = sum(news)
        wide = torch.randn((total, hkv * group + 3, dim), generator=g, dtype=torch.float64).to(self.kind)
        self.wide = wide.cuda()
        self.q = self.wide[:, 2:2 + hkv * group]
        self.k, self.v = k.to(self.kind).cuda(), v.to(self.kind).cuda()
        self.k64, self.v64, self.q64 = (x.double().cpu().numpy() for x in (self.k, self.v, self.q))

    def needed(self, n, m, t):
        """Whether one of the sequence's new tokens sees token t."""
        return t < n and m > 0 and (t < self.sinks or t > n - m - self.window)

    def run(self, max_seq_len=None, out=None, **kw):
        import torch

        from paper_2412_15803_amd import wq

        total, hq, dim = self.q.shape
        if out is None:
            out = torch.full((total, hq + 1, dim), 7.0, dtype=self.kind, device="cuda")[:, :hq]
        wq.window_attention(self.q, self.k, self.v, ints(self.table), ints(self.lens), out, self.scale, max_seq_len or max(max(self.lens), 1), self.window,
                            sinks=self.sinks, q_starts=None if self.starts is None else ints(self.starts), max_query_len=max(max(self.news), 1), **kw)
        torch.cuda.synchronize()
        return out

    def check(self, out):
        want, size, most = window_model.attend(self.q64, self.k64, self.v64, self.table, self.lens, self.starts, self.scale, self.window, self.sinks)
        assert most <= 60.0
        got = out.double().cpu().numpy()
        assert np.isfinite(got).all()
        off = np.abs(got - want) / (BOUND[self.dtype] * size + 1e-6)
        assert off.max() <= 1.0, (float(off.max()), np.unravel_index(off.argmax(), off.shape))
        return float(off.max())


def both(*cases):
    return [(d,) + c for c in cases for d in ("float16", "bfloat16")]


# lens, news, hkv, group, dim, page, window, sinks
STEPS = [
    ([1], [1], 1, 1, 64, 16, 10, 0), ([1, 2, 31, 32, 33, 64, 65], [1] * 7, 2, 3, 128, 16, 1000, 0), ([700], [1], 2, 4, 64, 16, 512, 4),
    ([300, 5, 1200, 77], [1] * 4, 2, 8, 128, 16, 100, 4), ([2000, 3000, 100], [1] * 3, 1, 16, 128, 32, 1500, 33), ([513, 64, 1], [1] * 3, 8, 1, 64, 8, 40, 1),
    ([257, 256, 255], [1] * 3, 1, 5, 128, 64, 1, 0), ([100, 90], [1, 1], 2, 2, 64, 1, 37, 3), ([100, 90], [1, 1], 2, 2, 128, 4, 64, 70), ([90, 300], [1, 1], 1, 7, 64, 2, 5, 0),
    ([5000], [1], 1, 2, 128, 1024, 5000, 0), ([9000, 4000, 40, 8000], [1] * 4, 2, 3, 128, 16, 100000, 0), ([60, 70], [1, 1], 1, 1, 64, 16, 0, 5), ([40], [1], 1, 2, 64, 16, 0, 0),
    ([50, 0, 20], [1, 0, 1], 2, 4, 64, 16, 16, 2), ([30] * 90, [1] * 90, 1, 2, 64, 16, 12, 3), ([1500] * 70, [1] * 70, 4, 2, 64, 16, 1400, 3),
]
FEWS = [  # several new tokens, up to 16 rows
    ([40, 41], [4, 3], 2, 4, 128, 16, 20, 3), ([1000, 3, 500], [2, 3, 5], 1, 3, 64, 16, 300, 4), ([2500], [16], 1, 1, 128, 16, 64, 0), ([17], [2], 1, 8, 64, 8, 4, 1),
    ([3000, 2], [2, 2], 2, 8, 128, 2, 2900, 0),
]
PROMPTS = [
    ([20], [20], 1, 1, 64, 16, 100, 0), ([33], [33], 1, 16, 64, 16, 9, 2), ([200], [200], 2, 4, 128, 16, 1000, 0), ([300], [300], 1, 3, 128, 16, 50, 4), ([257], [130], 2, 2, 64, 32, 64, 70),
    ([500, 3, 70, 129], [100, 3, 70, 1], 2, 4, 128, 16, 90, 4), ([130, 1], [129, 1], 1, 7, 64, 8, 200, 0), ([100, 90], [60, 90], 1, 2, 128, 1, 30, 3), ([90, 100], [90, 50], 2, 1, 64, 4, 100, 0),
    ([1500], [40], 2, 4, 128, 16, 100000, 0), ([3000, 2000], [17, 5], 1, 8, 64, 16, 2500, 5), ([640], [640], 1, 2, 128, 64, 128, 64), ([100], [100], 1, 4, 64, 16, 0, 5),
    ([100], [100], 1, 4, 64, 16, 0, 0), ([100], [100], 2, 2, 128, 16, 1, 0), ([60, 0, 300], [60, 0, 200], 1, 4, 64, 1024, 33, 1), ([40] * 70, [9] * 70, 1, 2, 64, 16, 12, 3),
]


@pytest.mark.parametrize("dtype,lens,news,hkv,group,dim,page,window,sinks", both(*STEPS, *FEWS, *PROMPTS))
def test_against_the_definition(dtype, lens, news, hkv, group, dim, page, window, sinks):
    require_gpu()
    announce(f"window {dtype} lens={lens[:4]} news={news[:4]} hkv={hkv} g={group} d={dim} page={page} w={window} s={sinks}")
    c = Case(sum(lens) + window, dtype, lens, news, hkv, group, dim, page, window, sinks)
    print("largest share of the bound", c.check(c.run()))


@pytest.mark.parametrize("seed", range(24))
def test_random_shapes(seed):
    require_gpu()
    rng = np.random.default_rng(seed)
    top = int(rng.choice([30, 200, 900]))
    lens = rng.integers(1, top + 1, rng.integers(1, 7)).tolist()
    news = [int(rng.integers(0, min(n, rng.choice([1, 6, 1000])) + 1)) for n in lens]
    news[0] = max(1, news[0])
    dtype = str(rng.choice(["float16", "bfloat16"]))
    args = (lens, news, int(rng.choice([1, 2, 3])), int(rng.integers(1, 17)), int(rng.choice([64, 128])), int(rng.choice([1, 4, 8, 16, 32])),
            int(rng.integers(0, top + 1)), int(rng.choice([0, 4, rng.integers(0, 150)])))
    announce(f"window {dtype} {args}")
    c = Case(seed, dtype, *args)
    c.check(c.run(max_seq_len=top + int(rng.integers(0, 500))))


@pytest.mark.parametrize("scale", [0.0, -0.09, 2.0 ** -10])
@pytest.mark.parametrize("news", [1, 80])
def test_scales(scale, news):
    require_gpu()
    c = Case(7, "float16", [150], [news], 2, 2, 128, 16, 60, 4, scale=scale)
    c.check(c.run())


@pytest.mark.parametrize("news", [1, 3, 90])
def test_uniform_weights_are_exact(news):
    """With equal keys, a power of two of visible tokens and small integers as values, the mean is exact in any order."""
    import torch

    require_gpu()
    c = Case(3, "float16", [200], [news], 2, 2, 64, 16, 32, 0, values="integers")
    c.k[:] = 0.5
    c.k64[:] = 0.5
    got = c.run().double().cpu().numpy()
    want, _, _ = window_model.attend(c.q64, c.k64, c.v64, c.table, c.lens, c.starts, c.scale, 32, 0)
    assert np.array_equal(got, torch.tensor(want).half().double().numpy())


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("news", [1, 4, 70])
def test_one_key_that_outweighs_the_rest(dtype, news):
    """Scores up to 300, so that sums of shifted weights would overflow unshifted: the chosen value comes out exactly."""
    require_gpu()
    c = Case(5, dtype, [190], [news], 1, 2, 128, 16, 100, 2, scale=1.0)
    c.k[:] = 0.0
    page = int(c.table[0][140 // 16])
    c.k[page, :, 140 % 16] = 8.0
    c.q[:] = 0.25
    got = c.run().double().cpu().numpy()
    want = c.v64[page, 0, 140 % 16]
    first = 190 - news
    for row in range(news):
        if first + row >= 140:
            assert np.array_equal(got[row], np.broadcast_to(want, got[row].shape))


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("news,group", [(1, 4), (5, 3), (16, 1), (100, 2), (128, 4)])
@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
def test_what_is_not_finite_reaches_only_rows_that_see_it(dim, news, group, value):
    """In a value and in a key: rows that do not see the token keep their bits."""
    import torch

    require_gpu()
    n, window, sinks, page = 300, 60, 3, 16
    c = Case(9, "float16", [n], [news], 2, group, dim, page, window, sinks)
    clean = c.run()
    first = n - news
    for t in sorted({1, first - window + 1, first, max(first - 3, 0), n - 1, n - 2, first - window // 2}):
        if c.table[0][t // page] < 0:
            continue
        for cache in (c.v, c.k):
            p = int(c.table[0][t // page])
            saved = cache[p, 1, t % page].clone()
            cache[p, 1, t % page, 5] = value
            got = c.run()
            cache[p, 1, t % page] = saved
            for row in range(news):
                place = first + row
                sees = t <= place and (t < sinks or t > place - window)
                assert torch.equal(got[row, :group], clean[row, :group])  # the other kv head
                mine, base = got[row, group:], clean[row, group:]
                if not sees:
                    assert torch.equal(mine, base), (t, row)
                elif cache is c.v:
                    assert not bool(torch.isfinite(mine[:, 5]).any())
                    assert torch.equal(mine[:, 6:], base[:, 6:])
                    if not math.isnan(value):
                        assert bool((mine[:, 5] == value).all())


def test_invalid_sequences_give_nan_and_leave_the_others_alone():
    import torch

    require_gpu()
    for news in ([1, 1, 1, 1, 1], [2, 2, 2, 2, 2], [40, 1, 40, 3, 40]):
        c = Case(13, "float16", [100, 100, 100, 100, 100], news, 2, 4, 64, 16, 50, 4)
        clean = c.run()
        starts = np.concatenate([[0], np.cumsum(news)])
        wrong = [(1, "lens", -3), (1, "lens", 0), (3, "lens", 101), (2, "lens", 1 << 30), (1, "page", 1 << 30), (4, "page", -1), (0, "page", c.k.shape[0])]
        for s, what, v in wrong:
            saved = c.lens[s], c.table[s].copy()
            if what == "lens":
                c.lens[s] = v
            else:
                c.table[s, 99 // 16] = v
            got = c.run(max_seq_len=100)
            c.lens[s], c.table[s] = saved
            for t in range(5):
                mine = slice(starts[t], starts[t + 1])
                if t != s:
                    assert torch.equal(got[mine], clean[mine]), (s, what, v, t)
                elif what == "lens":
                    assert bool(torch.isnan(got[mine]).all()), (s, what, v)
                else:
                    assert bool(torch.isnan(got[starts[t + 1] - 1]).all()), (s, what, v)


def test_starts_out_of_range_and_too_many_queries():
    import torch

    from paper_2412_15803_amd import wq

    require_gpu()
    c = Case(21, "float16", [60, 60, 60], [20, 20, 20], 1, 2, 64, 16, 100, 0)
    clean = c.run()
    c.starts = np.array([0, 20, 10, 60])  # falls; then a sequence of 50, more than max_query_len
    got = c.run()
    assert torch.equal(got[:10], clean[:10])
    assert bool(torch.isnan(got[20:60]).all())  # rows 10 to 20 belong to two sequences
    c.starts = np.array([-5, 20, 40, 61])
    got = c.run()
    assert bool((got[:20] == 7.0).all()) and torch.equal(got[20:40], clean[20:40]) and bool((got[40:] == 7.0).all())
    # All sequences few by max_query_len, one that is not.
    out = torch.full((60, 2, 64), 7.0, dtype=torch.float16, device="cuda")
    wq.window_attention(c.q, c.k, c.v, ints(c.table), ints(c.lens), out, c.scale, 60, 100, q_starts=ints([0, 8, 10, 60]), max_query_len=8)
    assert not bool(torch.isnan(out[:10]).any()) and bool(torch.isnan(out[10:]).all())


@pytest.mark.parametrize("news", [1, 50])
def test_offsets_beyond_32_bits(news):
    import torch

    from paper_2412_15803_amd import wq

    require_gpu()
    hkv, page, dim = 8, 16, 128
    pages = (5 << 30) // (hkv * page * dim * 2)
    k = torch.zeros((pages, hkv, page, dim), dtype=torch.float16, device="cuda")
    v = torch.zeros_like(k)
    c = Case(2, "float16", [100], [news], hkv, 2, dim, page, 64, 4)
    table = np.full_like(c.table, -1)
    for e, p in enumerate(c.table[0]):
        if p >= 0:
            table[0, e] = pages - 1 - e
            k[pages - 1 - e], v[pages - 1 - e] = c.k[int(p)], c.v[int(p)]
    want = c.run()
    out = torch.empty_like(want)
    wq.window_attention(c.q, k, v, ints(table), ints(c.lens), out, c.scale, 100, 64, sinks=4, q_starts=None if c.starts is None else ints(c.starts), max_query_len=news)
    assert torch.equal(out, want)


def test_page_order_does_not_matter():
    import torch

    require_gpu()
    for news in ([1, 1], [1, 90]):
        c = Case(31, "bfloat16", [700, 333], news, 2, 4, 128, 16, 400, 4)
        want = c.run()
        perm = torch.randperm(c.k.shape[0], generator=torch.Generator().manual_seed(1))
        k, v = torch.empty_like(c.k), torch.empty_like(c.v)
        k[perm.cuda()], v[perm.cuda()] = c.k, c.v
        c.k, c.v = k, v
        c.table = np.where(c.table >= 0, perm.numpy()[np.maximum(c.table, 0)], -1)
        assert torch.equal(c.run(), want)


def test_full_window_equals_decode_attention():
    """The same operation as paged_attention when the window covers everything."""
    import torch

    from paper_2412_15803_amd import wq

    require_gpu()
    c = Case(17, "float16", [900, 31, 4000], [1, 1, 1], 2, 4, 128, 16, 1 << 20, 0)
    got, other = c.run(), torch.empty((3, 8, 128), dtype=torch.float16, device="cuda")
    wq.paged_attention(c.q.contiguous(), torch.nan_to_num(c.k), torch.nan_to_num(c.v), ints(c.table), ints(c.lens), other, c.scale, 4000)
    assert float((got.float() - other.float()).abs().max()) < 5e-3 * float(other.float().abs().max())


def test_in_a_graph_on_another_stream():
    import torch

    from paper_2412_15803_amd import wq

    require_gpu()
    c = Case(23, "float16", [2500, 300, 90], [1, 30, 1], 2, 4, 64, 16, 2000, 4)
    table, lens, starts = ints(c.table), ints(c.lens), ints(c.starts)
    q = c.q.clone()
    out = torch.empty_like(q)
    work = wq.window_workspace(q, 2, 3, 2500, 2000, 4, 30)

    def call():
        wq.window_attention(q, c.k, c.v, table, lens, out, c.scale, 2500, 2000, sinks=4, q_starts=starts, max_query_len=30, workspace=work)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            call()
        for replay in range(6):
            q.copy_(c.q * (1 + replay))
            graph.replay()
            side.synchronize()
            got = out.clone()
            call()
            assert torch.equal(got, out)
    torch.cuda.synchronize()


@pytest.mark.parametrize("tokens,splits", [(17, False), (200, True)])
def test_one_sequence_with_fewer_new_tokens_than_rows(tokens, splits):
    """A buffer of rows that is not full: the sequence's rows are computed, few or many, and the rest is not written."""
    import torch

    from paper_2412_15803_amd import wq

    require_gpu()
    lens = 4000 if splits else 300
    for news in (1, 2, 4, 16, 17):
        c = Case(41, "float16", [lens], [news], 2, 4, 64, 16, 5000, 4)
        q = torch.cat([c.q, torch.zeros((tokens - news, 8, 64), dtype=c.kind, device="cuda")])
        out = torch.full_like(q, 7.0)
        wq.window_attention(q, c.k, c.v, ints(c.table), ints(c.lens), out, c.scale, lens, 5000, sinks=4, q_starts=ints([0, news]), max_query_len=tokens)
        c.check(out[:news])
        assert bool((out[news:] == 7.0).all())


def test_a_sequence_beyond_the_query_bound_is_nan_in_every_row():
    """Its rows are more than the launch has tiles for; the sequences after it keep theirs."""
    import torch

    from paper_2412_15803_amd import wq

    require_gpu()
    c = Case(43, "float16", [900, 100, 60], [900, 100, 30], 1, 4, 64, 16, 2000, 0)
    clean = c.run()
    out = torch.full((1030, 4, 64), 7.0, dtype=torch.float16, device="cuda")
    wq.window_attention(c.q, c.k, c.v, ints(c.table), ints(c.lens), out, c.scale, 900, 2000, q_starts=ints(c.starts), max_query_len=100)
    assert bool(torch.isnan(out[:900]).all())
    c.check(torch.cat([clean[:900], out[900:]]))


def test_without_a_workspace_on_another_stream():
    """The memory of a workspace made in the call belongs to the stream that the call is queued on."""
    import torch

    require_gpu()
    c = Case(47, "float16", [3000, 2500], [1, 1], 2, 4, 64, 16, 4000, 0)
    want = c.run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    outs = []
    for _ in range(20):
        out = torch.empty_like(want)
        side.wait_stream(torch.cuda.current_stream())
        c.run(out=out, stream=side)
        outs.append(out)
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)
