"""The choice of a word by chance where masks, temperatures and random numbers are extreme."""

import math

import numpy as np
import pytest
import torch

import sample_model as sm
from gpu_util import require_gpu
from paper_2412_15803_amd import wq
from test_gpu_sample import OPTIONS, TYPES, call, compare, fp32

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True, scope="module")
def _gpu():
    require_gpu()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("mask", ["lowest", -10000.0])
@pytest.mark.parametrize("rows", [1, 12, 90])
def test_beginnings_masked_by_a_large_negative_number(dtype, mask, rows):
    """What all chunks' bins refer to is no logit of the words that can be chosen."""
    rng = np.random.default_rng(rows)
    vocab = 30011 if rows < 50 else 9001
    value = torch.finfo(dtype).min if mask == "lowest" else mask
    options = [OPTIONS[i % len(OPTIONS)] for i in range(3, 3 + rows)]
    logits = torch.from_numpy(rng.standard_normal((rows, vocab)) * 3).to(dtype).cuda()
    logits[:, :8700] = value
    logits[:, 8800:8900] = value
    logits[0, 8700:-1] = value  # one word is left
    compare(logits, options, rng, tries=2)


@pytest.mark.parametrize("dtype", TYPES)
def test_small_temperatures(dtype):
    """The best words lie in the last chunk, beyond what the bins refer to."""
    rng = np.random.default_rng(5)
    temperatures = [1e-2, 1e-4, 1e-8, 1e-12, 1e-14, 1e-16, 1e-20, 1e-30, 1e-37]
    settings = [dict(), dict(top_k=40), dict(top_p=0.7), dict(min_p=0.9), dict(top_k=40, top_p=0.9)]
    options = [dict(temperature=t, **o) for t in temperatures for o in settings]
    logits = torch.from_numpy(rng.standard_normal((len(options), 20011))).to(dtype).cuda()
    logits[:, 19000] = 9.25
    logits[::2, 10000] = 9.25  # with an equal in another chunk
    compare(logits, options, rng, tries=1)


@pytest.mark.parametrize("scale,temperature", [(1e6, 1e6), (1e6, 1.0), (1e30, 1e30), (1e30, 1.0), (3e37, 1e-20), (1e-30, 1e-30), (1e-20, 1.0)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_logits_of_any_size(dtype, scale, temperature):
    rng = np.random.default_rng(4)
    settings = [dict(), dict(top_k=40), dict(top_p=0.7), dict(min_p=0.3), dict(top_k=9000, top_p=0.9)]
    options = [dict(temperature=temperature, **o) for o in settings]
    logits = torch.from_numpy(rng.standard_normal((len(options), 10007)) * scale).to(dtype).cuda()
    compare(logits, options, rng, tries=2)


def test_the_largest_random_number():
    """The weights' sum over a chunk and the sum that is made of its words one by one differ by their roundings:
    4096 words weigh 16000.4 steps each, which is 16000 word by word, and the random number falls behind them."""
    steps = 2.0 ** 48  # of a vocabulary of 16384 words
    logits = torch.full((1, 16384), -200.0, device="cuda")
    logits[0, 0] = 0.0
    logits[0, 8192:12288] = math.log(8000.4 / steps)  # half of these is left out
    logits[0, 12288:] = math.log(16000.4 / steps)
    option = dict(top_p=float(np.float32(1 - 2.0 ** -24)))
    weights = sm.stays(list(logits[0].double().cpu().numpy()), **fp32(option))
    assert 4096 < np.count_nonzero(weights) < 8193
    for u in (1.0, math.inf):
        token, share = call(logits, [u], [option])
        assert token[0] >= 8192 and weights[token[0]] > 0
        assert abs(share[0] - weights[token[0]] / weights.sum()) <= 1e-3 * share[0]


@pytest.mark.parametrize("rows", [1, 100])
@pytest.mark.parametrize("vocab", [20011, 128256])
def test_the_largest_random_number_of_any_row(rows, vocab):
    """Every row has a word, whatever the random number."""
    g = torch.Generator(device="cuda").manual_seed(rows)
    logits = torch.randn((rows, vocab), generator=g, device="cuda") * 4
    token = torch.full((rows,), -7, dtype=torch.int32, device="cuda")
    for p in (None, 0.3, 0.99, 0.9999999):
        top_p = None if p is None else torch.full((rows,), p, device="cuda")
        for u in (0.0, 2.0 ** -149, 1 - 2.0 ** -24, 1.0):
            token.fill_(-7)
            wq.sample_logits(logits, torch.full((rows,), u, device="cuda"), token, top_p=top_p)
            assert bool(((token >= 0) & (token < vocab)).all())
