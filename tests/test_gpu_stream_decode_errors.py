"""The decoding example says when its pool is too small and when no word is
allowed."""

from __future__ import annotations

import numpy as np
import pytest

from gpu_util import announce, require_gpu

pytestmark = pytest.mark.gpu

WORDS = (5, 90, 33)  # 1 + 6 + 3 pages of 16, each with a partly filled last one


def prompts_of(model):
    rng = np.random.default_rng(4)
    return [rng.integers(0, model.vocab, n).tolist() for n in WORDS]


@pytest.mark.parametrize("pages,samples,steps,what", [(9, 1, 4, "prompts"), (9, 2, 4, "prompts"), (12, 2, 4, "forks"), (13, 2, 40, "steps"), (10, 1, 40, "steps")])
def test_a_pool_that_is_too_small(pages, samples, steps, what):
    from paper_2412_15803_amd import stream_decode as sd

    require_gpu()
    announce(f"stream pool of {pages} pages, {samples} samples: too small for the {what}")
    model = sd.Decoder()
    with pytest.raises(RuntimeError, match="pages"):
        sd.generate(model, prompts_of(model), samples, steps, 1000, 0, pages=pages)


def test_a_pool_that_just_fits():
    from paper_2412_15803_amd import stream_decode as sd

    require_gpu()
    model = sd.Decoder()
    sd.generate(model, prompts_of(model), 2, 4, 1000, 0, pages=13)  # 5, 90 and 33 words: four more fit their pages
    sd.generate(model, prompts_of(model), 1, 4, 1000, 0, pages=10)


def test_no_word_allowed():
    import torch

    from paper_2412_15803_amd import stream_decode as sd

    require_gpu()
    model = sd.Decoder()
    allowed = torch.zeros((1, -(-model.vocab // 32)), dtype=torch.int32, device="cuda")
    with pytest.raises(RuntimeError, match="word"):
        sd.generate(model, prompts_of(model), 2, 4, 1000, 0, allowed=allowed)
