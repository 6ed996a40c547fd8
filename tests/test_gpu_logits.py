"""GPU tests of the step from logits to a token against the 64-bit model.

Two kinds of inputs.  On exact ones (small integers, penalties that are powers of
two) every fp32 operation is exact, so values and tokens are compared bit for
bit.  On random ones each of at most five fp32 operations rounds once, by at most
2^-24 of the largest magnitude it meets, and the result is rounded once to the
logits' type."""

from __future__ import annotations

import math

import numpy as np
import pytest

import logits_model
from gpu_util import announce, require_gpu

pytestmark = pytest.mark.gpu

TYPES = ("float16", "bfloat16", "float32")
STEP = {"float16": 2.0 ** -11, "bfloat16": 2.0 ** -8, "float32": 2.0 ** -24}
TINY = {"float16": 2.0 ** -25, "bfloat16": 0.0, "float32": 0.0}  # half the least subnormal


def ints(a):
    import torch

    return torch.from_numpy(np.ascontiguousarray(np.asarray(a, dtype=np.int32))).cuda()


def floats(a):
    import torch

    return torch.tensor(np.asarray(a, dtype=np.float32)).cuda()


def packed_mask(allowed):
    rows, vocab = allowed.shape
    words = -(-vocab // 32)
    bits = np.zeros((rows, words * 32), dtype=np.uint64)
    bits[:, :vocab] = allowed
    return (bits.reshape(rows, words, 32) << np.arange(32, dtype=np.uint64)).sum(-1).astype(np.uint32).view(np.int32)


def case(seed, rows, vocab, history, bias, allow, exact):
    rng = np.random.default_rng(seed)
    x = rng.integers(-30, 31, (rows, vocab)).astype(np.float64) if exact else rng.normal(0, 4, (rows, vocab))
    c = dict(x=x, allowed=rng.random((rows, vocab)) < allow, rows=rows, vocab=vocab)
    if history:
        c.update(history=rng.integers(0, max(1, min(vocab, 1 + history // 3)), (rows, history)).astype(np.int32) * max(1, vocab // (1 + history)),
                 lens=rng.integers(0, history + 1, rows), prompts=rng.integers(0, history + 1, rows))
        pick = (lambda s: rng.choice(s, rows)) if exact else (lambda s: rng.uniform(min(s), max(s), rows).astype(np.float32))
        c.update(repetition=pick([1.0, 2.0, 0.5]), frequency=pick([0.0, 0.25, 1.0]), presence=pick([0.0, 0.5, -2.0]))
    if bias:
        c.update(ids=rng.integers(0, vocab, (rows, bias)), values=rng.integers(-40, 41, (rows, bias)).astype(np.float64) if exact
                 else rng.normal(0, 10, (rows, bias)).astype(np.float32).astype(np.float64), blens=rng.integers(0, bias + 1, rows))
    return c


def run(c, dtype, pad=0, out_pad=0, off=0, in_place=False, with_token=True, mask_pad=0):
    import torch

    from paper_2412_15803_amd import wq

    kind = getattr(torch, dtype)
    wide = torch.full((c["rows"], off + c["vocab"] + pad), 7.0, dtype=kind, device="cuda")
    x = wide[:, off:off + c["vocab"]]
    x.copy_(torch.from_numpy(c["x"]))
    given = x.double().cpu().numpy()  # the values that the type holds
    if in_place:
        y = x
    else:
        wide_out = torch.full((c["rows"], off + c["vocab"] + out_pad), 9.0, dtype=kind, device="cuda")
        y = wide_out[:, off:off + c["vocab"]]
    token = torch.full((c["rows"],), -7, dtype=torch.int32, device="cuda") if with_token else None
    packed = packed_mask(c["allowed"])
    mask = ints(np.pad(packed, ((0, 0), (0, mask_pad))))[:, :packed.shape[1]]
    more = {}
    if "history" in c:
        more.update(history=ints(c["history"]), history_lens=ints(c["lens"]), prompt_lens=ints(c["prompts"]), repetition=floats(c["repetition"]),
                    frequency=floats(c["frequency"]), presence=floats(c["presence"]))
    if "ids" in c:
        more.update(bias_ids=ints(c["ids"]), bias_values=floats(c["values"]), bias_lens=ints(c["blens"]))
    wq.process_logits(x, y, token=token, mask=mask, **more)
    torch.cuda.synchronize()
    if pad:
        assert bool((wide[:, off + c["vocab"]:] == 7.0).all())
    if out_pad and not in_place:
        assert bool((wide_out[:, off + c["vocab"]:] == 9.0).all()) and bool((wide_out[:, :off] == 9.0).all())
    return given, y.double().cpu().numpy(), None if token is None else token.tolist()


def model(c, given):
    outs, words = [], []
    for i in range(c["rows"]):
        kw = {}
        if "history" in c:
            kw.update(history=c["history"][i, :c["lens"][i]].tolist(), prompt=c["prompts"][i], repetition=float(c["repetition"][i]),
                      frequency=float(c["frequency"][i]), presence=float(c["presence"][i]))
        if "ids" in c:
            n = c["blens"][i]
            kw["bias"] = list(zip(c["ids"][i, :n].tolist(), c["values"][i, :n].tolist()))
        v, w = logits_model.process(given[i].tolist(), c["allowed"][i], **kw)
        outs.append(v)
        words.append(w)
    return np.array(outs), words


SHAPES = [(1, 1, 0, 0, 1.0), (1, 1, 3, 2, 1.0), (3, 33, 5, 3, 0.5), (2, 500, 64, 10, 0.02), (5, 2049, 300, 7, 0.4), (2, 8209, 1000, 300, 0.9),
          (1, 128256, 600, 8, 0.02), (3, 50257, 3001, 0, 0.5), (17, 4099, 0, 31, 0.3), (2, 4096, 17, 1, 0.0), (300, 4100, 90, 4, 0.6)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", SHAPES)
def test_exact_inputs_bit_for_bit(dtype, shape):
    import torch

    require_gpu()
    announce(f"logits {dtype} {shape}")
    c = case(sum(shape[:4]), *shape, exact=True)
    given, got, words = run(c, dtype)
    want, best = model(c, given)
    want = torch.tensor(want).to(getattr(torch, dtype)).double().numpy()
    assert np.array_equal(got, want)
    assert words == best


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", SHAPES)
def test_random_inputs(dtype, shape):
    require_gpu()
    c = case(sum(shape[:4]) + 1, *shape, exact=False)
    given, got, words = run(c, dtype)
    want, best = model(c, given)
    allowed = c["allowed"]
    assert np.all(got[~allowed] == -math.inf)
    # Magnitudes stay below what the terms add up to: |x| r + f c + |p| + |b|.
    counts = np.zeros_like(want)
    if "history" in c:
        for i in range(c["rows"]):
            np.add.at(counts[i], c["history"][i, :c["lens"][i]], 1)
    size = np.abs(given) * 2 + counts + 2 + (60 if "ids" in c else 0)
    bound = 5 * 2.0 ** -24 * size + STEP[dtype] * np.abs(np.where(allowed, want, 0)) * 1.0001 + TINY[dtype]
    assert np.all(np.abs(got - want)[allowed] <= bound[allowed])
    for i, w in enumerate(words):
        # The chosen word's exact value is within the rounding of the best one's.
        if best[i] < 0:
            assert w == -1
        else:
            assert allowed[i, w] and want[i, w] >= want[i, best[i]] - 10 * 2.0 ** -24 * (size[i, w] + size[i, best[i]])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("kw", [dict(pad=3, out_pad=3), dict(pad=1, out_pad=9), dict(off=1, pad=2, out_pad=2), dict(off=5, pad=4, out_pad=7),
                                dict(in_place=True, pad=5), dict(with_token=False), dict(mask_pad=2, pad=8, out_pad=16), dict(off=3, in_place=True)])
def test_rows_that_lie_apart_and_off_16_byte_boundaries(dtype, kw):
    import torch

    require_gpu()
    for vocab in (5, 2051, 5000):
        c = case(vocab, 4, vocab, 40, 6, 0.5, exact=True)
        given, got, words = run(c, dtype, **kw)
        want, best = model(c, given)
        assert np.array_equal(got, torch.tensor(want).to(getattr(torch, dtype)).double().numpy())
        assert words is None or words == best


@pytest.mark.parametrize("dtype", TYPES)
def test_special_values(dtype):
    """NaN never wins, -infinity wins only alone, infinities pass; a tie goes to the lowest word; a masked NaN or infinity stays out."""
    import torch

    from paper_2412_15803_amd import wq

    require_gpu()
    nan, inf = math.nan, math.inf
    rows = [[nan, -inf, -inf, nan], [nan] * 4, [1.0, 3.0, 3.0, nan], [inf, inf, 2.0, -inf], [nan, inf, 5.0, inf], [-inf] * 4, [0.0, -0.0, -1.0, 0.0]]
    allowed = np.ones((7, 4), dtype=bool)
    allowed[4] = [False, False, True, False]
    x = torch.tensor(rows, device="cuda").to(getattr(torch, dtype))
    out, token = torch.empty_like(x), torch.empty(7, dtype=torch.int32, device="cuda")
    wq.process_logits(x, out, token=token, mask=ints(packed_mask(allowed)))
    assert token.tolist() == [1, -1, 1, 0, 2, 0, 0]
    want = np.where(allowed, np.array(rows), -inf)
    assert np.array_equal(out.double().cpu().numpy(), want, equal_nan=True)
    wq.process_logits(x, out)  # nothing to do but a copy
    assert np.array_equal(out.double().cpu().numpy(), np.array(rows), equal_nan=True)


def test_ties_across_tiles_go_to_the_lowest_word():
    import torch

    from paper_2412_15803_amd import wq

    require_gpu()
    for rows, vocab in ((2, 100003), (700, 9001)):
        x = torch.zeros((rows, vocab), dtype=torch.float16, device="cuda")
        first = torch.arange(rows, device="cuda") * 13 % (vocab - 1)
        for at in (vocab - 1, vocab // 2, 1, 0):
            x[torch.arange(rows, device="cuda"), torch.clamp(first + at, max=vocab - 1)] = 5.0
        token = torch.empty(rows, dtype=torch.int32, device="cuda")
        wq.process_logits(x, torch.empty_like(x), token=token)
        assert token.tolist() == first.tolist()


def test_words_and_lengths_out_of_range_are_ignored():
    import torch

    from paper_2412_15803_amd import wq

    require_gpu()
    x = torch.full((3, 40), 8.0, device="cuda")
    history = ints([[-1, 40, 1 << 30, 3, -(1 << 31), 7]] * 3)
    out, token = torch.empty_like(x), torch.empty(3, dtype=torch.int32, device="cuda")
    wq.process_logits(x, out, token=token, history=history, history_lens=ints([99, -4, 4]), prompt_lens=ints([-3, 2, 99]), repetition=floats([2.0] * 3),
                      frequency=floats([1.0] * 3), bias_ids=ints([[40, -2, 5, 5, 0]] * 3), bias_values=floats([[50.0, 50.0, 9.0, 1.0, 100.0]] * 3),
                      bias_lens=ints([4, 99, -1]))
    want = np.full((3, 40), 8.0)
    want[0, [3, 7]] = 3.0
    want[0, 5], want[1, 5], want[1, 0] = 9.0, 9.0, 108.0
    want[2, 3] = 4.0
    assert np.array_equal(out.cpu().numpy(), want) and token.tolist() == [5, 0, 0]


def test_counts_beyond_16_bits():
    import torch

    from paper_2412_15803_amd import wq

    require_gpu()
    history = torch.full((1, 200001), 2, dtype=torch.int32, device="cuda")
    x = torch.zeros((1, 7), device="cuda")
    out = torch.empty_like(x)
    wq.process_logits(x, out, history=history, prompt_lens=ints([1]), frequency=floats([0.5]))
    assert out.tolist() == [[0, 0, -100000.0, 0, 0, 0, 0]]


def test_in_a_graph_on_another_stream():
    import torch

    from paper_2412_15803_amd import wq

    require_gpu()
    c = case(3, 4, 9000, 200, 12, 0.3, exact=True)
    x = torch.from_numpy(c["x"]).half().cuda()
    out, token = torch.empty_like(x), torch.empty(4, dtype=torch.int32, device="cuda")
    mask, history, lens = ints(packed_mask(c["allowed"])), ints(c["history"]), ints(c["lens"])
    work, rep = wq.logits_workspace(x), floats([2.0] * 4)

    def call():
        wq.process_logits(x, out, token=token, mask=mask, history=history, history_lens=lens, repetition=rep, workspace=work)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            call()
        for replay in range(6):
            x.copy_(x.roll(1 + replay, 1))
            graph.replay()
            side.synchronize()
            got, words = out.clone(), token.clone()
            call()
            assert torch.equal(got, out) and torch.equal(words, token)
    torch.cuda.synchronize()
