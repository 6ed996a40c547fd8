"""The operators together, as a server runs them: conversations decoded step by
step in a window (pages reserved, forked, given back, compacted) end with the
logits that the same words give as one prompt.

A word's logits depend on the cached keys and values only through attention, so
both ways compute the same function; they differ in the order of fp32 sums and in
where results are rounded to fp16.  Over two layers, each rounding (relative
2^-11 of values of order 1, a dozen of them on the way, amplified by the norms by
at most a few times) leaves the logits, of standard deviation about 1, within
0.05 of each other."""

from __future__ import annotations

import numpy as np
import pytest

from gpu_util import announce, require_gpu

pytestmark = pytest.mark.gpu


def as_one_prompt(model, words, window, sinks):
    import torch

    from paper_2412_15803_amd import stream_decode as sd

    cache = sd.Cache(model, 1, len(words), window, sinks)
    lens = torch.tensor([len(words)], dtype=torch.int32, device="cuda")
    cache.reserve(lens)
    starts = torch.tensor([0, len(words)], dtype=torch.int32, device="cuda")
    return model.forward(torch.tensor(words, dtype=torch.int32, device="cuda"), cache, lens, starts, len(words))[-1]


@pytest.mark.parametrize("samples,steps,window,sinks,page", [(1, 40, 1000, 0, 16), (2, 70, 32, 4, 16), (3, 50, 17, 0, 8), (2, 33, 24, 9, 32)])
def test_streaming_equals_one_prompt(samples, steps, window, sinks, page):
    import torch

    from paper_2412_15803_amd import stream_decode as sd

    require_gpu()
    announce(f"stream samples={samples} steps={steps} window={window} sinks={sinks} page={page}")
    model = sd.Decoder()
    rng = np.random.default_rng(steps)
    prompts = [rng.integers(0, model.vocab, n).tolist() for n in (5, 90, 33)]
    allowed = torch.full((1, -(-model.vocab // 32)), 0x7FFF7FFF, dtype=torch.int32, device="cuda")  # words 15 and 31 of every 32 are out
    history, lens, logits, cache = sd.generate(model, prompts, samples, steps, window, sinks, page, allowed, room=1)
    torch.cuda.synchronize()
    assert cache.shortfall.item() == 0
    slots = len(prompts) * samples
    for i in range(slots):
        words = history[i, :int(lens[i])].tolist()
        prompt = prompts[i if i < 3 else (i - 3) // (samples - 1)]
        assert words[:-steps] == prompt
        assert all(w % 32 not in (15, 31) for w in words[-steps:])
        want = as_one_prompt(model, words, window, sinks)
        off = float((logits[i].float() - want.float()).abs().max())
        assert off < 0.05 * max(1.0, float(want.float().std())), (i, off)
    # Only what the next word sees is still held, and every page by the table alone.
    held = torch.bincount(cache.table[cache.table >= 0].long(), minlength=cache.refs.numel())
    assert torch.equal(held.int(), cache.refs)
    for i in range(slots):
        n = int(lens[i])
        for e, p in enumerate(cache.table[i].tolist()):
            seen = any(t < sinks or t + window > n for t in range(e * page, e * page + page)) and e * page < n
            assert (p >= 0) == seen, (i, e)
    # Dropping and compacting leaves the others' next step as it is.
    other = torch.arange(1, slots, 2, dtype=torch.int32, device="cuda")
    new = lens + 1
    token = history[torch.arange(slots), (lens - 1).long()]
    cache.reserve(new)
    before = model.forward(token, cache, new, None, 1)
    cache.drop(torch.arange(0, slots, 2, dtype=torch.int32, device="cuda"))
    cache.compact()
    assert int(cache.table.max()) < int(cache.live) == int((cache.refs > 0).sum())
    keep = torch.zeros_like(new)
    keep[other.long()] = new[other.long()]
    after = model.forward(token, cache, keep, None, 1)
    assert torch.equal(after[other.long()], before[other.long()])


def test_command_runs(capsys):
    from paper_2412_15803_amd import stream_decode as sd

    require_gpu()
    sd.main(["--prompts", "2", "--steps", "8"])
    out = capsys.readouterr().out
    assert "words/s" in out and "pages" in out
