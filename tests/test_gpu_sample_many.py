"""The choice of a word by chance in large batches, whose plans, lists and choices have a launch each, and in batches
of several launches, against the model in float64."""

import math

import numpy as np
import pytest
import torch

import sample_model as sm
from gpu_util import require_gpu
from paper_2412_15803_amd import wq
from test_gpu_sample import OPTIONS, TYPES, call, fp32

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True, scope="module")
def _gpu():
    require_gpu()


def chunks(vocab, dtype):
    """Workgroups of a row: 8192 words each, wherever in 16 bytes it starts."""
    return -(-(vocab + (3 if dtype is torch.float32 else 7)) // 8192)


def compare(logits, options, rows, rng, tries=2):
    """The rows of `logits` with their options over and over, `rows` of them, each with a random number of its own that
    is clear of the borders.  More than 256 workgroups: the launches of large batches."""
    assert rows * chunks(logits.shape[1], logits.dtype) > 256
    x = logits.double().cpu().numpy()
    weights = [sm.stays(list(row), **fp32(o)) for row, o in zip(x, options)]
    n = len(options)
    some = np.arange(rows) % n
    wide = torch.full((rows, logits.shape[1] + 3), 60.0, dtype=logits.dtype, device="cuda")[:, :logits.shape[1]]
    wide.copy_(logits[torch.from_numpy(some).cuda()])
    for _ in range(tries):
        random = []
        for i in some:
            u = float(np.float32(rng.random()))
            while weights[i] is not None and not sm.clear_of_borders(weights[i], u):
                u = float(np.float32(rng.random()))
            random.append(min(u, 1 - 2.0 ** -24))
        token, share = call(wide, random, [options[i] for i in some])
        for r, i in enumerate(some):
            want, part = sm.choose(weights[i], random[r])
            assert token[r] == want, (r, options[i], random[r], token[r], want)
            assert abs(share[r] - part) <= 2.0 ** -23 * part + 1e-12, (r, options[i], share[r], part)


def normal(rng, rows, vocab, dtype, deviation=3):
    return torch.from_numpy(rng.standard_normal((rows, vocab)) * deviation).to(dtype).cuda()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab,rows", [(1, 300), (7, 1000), (500, 300), (4099, 301), (20011, 100), (33000, 60)])
def test_options(dtype, vocab, rows):
    rng = np.random.default_rng(vocab)
    options = OPTIONS + [dict(top_k=20), dict(top_k=70, min_p=0.02), dict(top_k=200, top_p=0.9), dict(top_k=260), dict(top_k=6000), dict(min_p=0.5, temperature=3.0)]
    compare(normal(rng, len(options), vocab, dtype), options, rows, rng)


@pytest.mark.parametrize("dtype", TYPES)
def test_a_large_vocabulary(dtype):
    rng = np.random.default_rng(8)
    options = [dict(), dict(top_k=50, top_p=0.95, temperature=0.8), dict(top_p=0.9), dict(min_p=0.05), dict(top_k=5000)]
    compare(normal(rng, len(options), 128256, dtype), options, 40, rng)


@pytest.mark.parametrize("dtype", TYPES)
def test_equal_logits(dtype):
    """Whole groups of equal words at the cut, in lists that hold them and in ones that do not."""
    rng = np.random.default_rng(6)
    values = np.array([-2.0, 0.0, -0.0, 1.5, 1.5, 3.0])
    for vocab, rows in ((2000, 270), (30000, 80)):
        options = OPTIONS + [dict(top_k=k) for k in (2, 100, 333, 1999, 4500, 20000)] + [dict(top_p=p) for p in (0.01, 0.5, 0.75)] + [dict(top_k=9000, top_p=0.6, min_p=0.3)]
        logits = torch.from_numpy(rng.choice(values, (len(options), vocab))).to(dtype).cuda()
        same = [dict(top_k=17), dict(top_p=0.7), dict(top_k=7000, top_p=0.5), dict(top_k=7000)]
        compare(torch.cat([logits, torch.full((len(same), vocab), -5.0, dtype=dtype, device="cuda")]), options + same, rows, rng)


@pytest.mark.parametrize("dtype", TYPES)
def test_long_lists(dtype):
    """Top-p behind a top-k of more words than a list holds, and cuts in bins that hold more."""
    rng = np.random.default_rng(12)
    options = [dict(top_k=5000, top_p=0.9), dict(top_k=15000, top_p=0.5, min_p=0.001), dict(top_k=9000, min_p=0.01), dict(top_p=0.97, temperature=5.0), dict(top_k=12000, temperature=4.0)]
    for deviation in (3, 0.02):
        compare(normal(rng, len(options), 20011, dtype, deviation), options, 100, rng)


@pytest.mark.parametrize("dtype", TYPES)
def test_words_that_take_no_part(dtype):
    rng = np.random.default_rng(7)
    logits = normal(rng, 11, 9001, dtype, 2)
    lowest = torch.finfo(dtype).min
    logits[0] = -math.inf
    logits[1] = math.nan
    logits[2] = -math.inf
    logits[2, 8999] = -3.0
    logits[3, ::2] = math.nan
    logits[4, 10:8990] = -math.inf
    logits[5, 77], logits[5, 8500] = math.inf, math.inf
    logits[6] = -math.inf
    logits[6, 9000] = math.inf
    logits[7, :100] = math.nan
    logits[8, :8900] = lowest
    logits[9, 50:] = lowest
    logits[10] = lowest
    options = [dict(), dict(top_k=5), dict(top_p=0.5), dict(top_k=20, top_p=0.9), dict(top_k=3000), dict(), dict(top_k=4, min_p=0.5), dict(temperature=0.0), dict(top_p=0.9),
               dict(top_k=40, top_p=0.999), dict(top_p=0.25)]
    compare(logits, options, 187, rng)
    for option in (dict(temperature=0.0), dict(top_k=6), dict(top_p=0.8), dict(top_k=30, top_p=0.8), dict(min_p=0.3)):
        compare(logits, [option] * 11, 187, rng, tries=1)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab,rows", [(100, 4100), (9000, 2053), (120000, 275)])
def test_batches_of_several_launches(dtype, vocab, rows):
    """More than 4096 workgroups: rows of a later launch have their own numbers, lists and results."""
    per = chunks(vocab, dtype)
    assert rows > 4096 // per
    rng = np.random.default_rng(rows)
    options = [dict(top_k=20, top_p=0.9, min_p=0.01, temperature=0.7), dict(top_p=0.8), dict(temperature=0.0), dict(top_k=30), dict(min_p=0.1), dict(), dict(top_k=500, temperature=1.5)]
    compare(normal(rng, len(options), vocab, dtype), options, rows, rng, tries=1)


def test_no_lists_at_all():
    """Nothing but random numbers, over several launches."""
    rng = np.random.default_rng(2)
    for rows, vocab in ((4200, 64), (300, 4099)):
        compare(normal(rng, 20, vocab, torch.float32), [dict()] * 20, rows, rng)


def test_small_and_large_batches_agree():
    """Rows by themselves, a few at a time and in a large batch: the same words and shares."""
    rng = np.random.default_rng(9)
    vocab, rows = 30011, 96
    logits = normal(rng, rows, vocab, torch.float16)
    options = [(OPTIONS + [dict(top_k=64), dict(top_k=9000, top_p=0.7)])[i % 14] for i in range(rows)]
    random = [float(np.float32(u)) for u in rng.random(rows)]
    large = call(logits, random, options)
    for size in (1, 7, 60):
        for i in range(0, rows, size):
            token, share = call(logits[i:i + size], random[i:i + size], options[i:i + size])
            assert token == large[0][i:i + size] and np.allclose(share, large[1][i:i + size], rtol=2.0 ** -22, atol=0)


def test_captured_and_replayed():
    rows, vocab = 320, 9001
    logits = torch.zeros((rows, vocab), dtype=torch.bfloat16, device="cuda")
    random, p, t = torch.zeros(rows, device="cuda"), torch.full((rows,), 0.9, device="cuda"), torch.full((rows,), 0.8, device="cuda")
    m = torch.full((rows,), 0.01, device="cuda")
    k = (torch.arange(rows, device="cuda", dtype=torch.int32) % 4) * 40
    token, share = torch.empty(rows, dtype=torch.int32, device="cuda"), torch.empty(rows, device="cuda")
    workspace = wq.sample_workspace(logits)

    def step():
        wq.sample_logits(logits, random, token, temperature=t, top_k=k, top_p=p, min_p=m, share=share, workspace=workspace)

    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in range(4):
        g = torch.Generator(device="cuda").manual_seed(seed)
        logits.copy_(torch.randn(logits.shape, generator=g, device="cuda") * 3)
        random.copy_(torch.rand(rows, generator=g, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        kept = token.clone(), share.clone()
        token.fill_(-9)
        step()
        assert torch.equal(kept[0], token) and torch.equal(kept[1], share) and int(token.min()) >= 0


@pytest.mark.parametrize("vocab,options", [
    (262144, [dict(top_p=0.95, temperature=2.0), dict(top_p=0.9), dict(top_k=50, top_p=0.95), dict(top_k=30000, min_p=0.001)]),
    (1 << 20, [dict(top_p=0.95, temperature=2.0), dict(top_k=200, temperature=0.9)])])
def test_the_largest_vocabularies(vocab, options):
    """Up to the largest that there may be; cuts in bins of more words than a list holds among them."""
    rng = np.random.default_rng(vocab)
    compare(normal(rng, len(options), vocab, torch.float32), options, 9, rng)
