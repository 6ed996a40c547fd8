"""Random numbers and shares of the probability that fall exactly on a border between words: the sums of equal weights
and their parts are whole numbers of steps, so the word is the exact one there too."""

import pytest
import torch

from gpu_util import require_gpu
from test_gpu_sample import TYPES, call

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True, scope="module")
def _gpu():
    require_gpu()


PARTS = [0.0, 2.0 ** -12, 0.125, 0.25, 0.375, 0.5, 0.75, 0.875, 1 - 2.0 ** -12]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab,times", [(96, 1), (4096, 1), (4096, 40), (28672, 1), (28672, 3), (122880, 1)])
@pytest.mark.parametrize("value,temperature", [(-5.0, 1.0), (3.25, 0.7), (0.0, 1.0)])
def test_equal_words(dtype, vocab, times, value, temperature):
    """n equal words, of which top-p leaves the first ceil(top_p n): the word is floor(random n) of those that stay."""
    logits = torch.full((len(PARTS) * times, vocab), value, dtype=dtype, device="cuda")
    random = PARTS * times
    for top_p in (1.0, 0.5, 0.25, 0.6875):
        for top_k in (0, 64, vocab // 8 * 5):
            n = -(-(top_k or vocab) * 16 * top_p // 16)
            token, share = call(logits, random, [dict(top_p=top_p, top_k=top_k, temperature=temperature)] * len(random))
            assert token == [int(u * n) for u in random], (top_p, top_k)
            assert all(abs(s * n - 1) <= 2.0 ** -23 for s in share)


@pytest.mark.parametrize("rows", [1, 300])
def test_twice_as_many(rows):
    """Four words of the largest logit, and others that weigh nothing beside them."""
    logits = torch.full((rows, 5000), -2000.0, device="cuda")
    logits[:, [7, 1000, 3000, 4999]] = 1.7
    for u, p, want in ((0.5, 1.0, 3000), (0.25, 1.0, 1000), (0.5 - 2.0 ** -25, 1.0, 1000), (0.0, 1.0, 7), (0.5, 0.5, 1000), (0.5, 0.75, 1000), (2.0 / 3, 0.75, 3000), (0.5, 0.25, 7)):
        token, _ = call(logits, [u] * rows, [dict(top_p=p)] * rows)
        assert token == [want] * rows, (u, p)
